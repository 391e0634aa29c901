// Orthogonalising an update by Newton-Schulz products (batches of rows x cols matrices):
//
//   X = G / (||G||_F + eps);  `steps` times: A = X X^T, X <- a X + (b A + c A A) X      (rows <= cols)
//                                            A = X^T X, X <- X (a + b A + c A A)        (rows > cols: the same X)
//
// so that A is square in the smaller size and X is never transposed. Every product runs on the fp16 matrix cores with
// each factor held as two fp16 parts (KIND_SPLIT of tile.h), which keeps fp32's exactness at 3 fp16 products each.
// A and A A are symmetric: only blocks on and above the diagonal are computed, and written to both places.
// Each step is three launches; their epilogues apply a, b, c and write the next factor in its two parts. Where A has
// blocks for few CUs (a small side against a long one) its k is split and a fourth launch joins the sums. Small
// matrices are one launch in all (k_small).
//
// Measured (five steps): 4096 x 4096 fp32 3.3 ms, 411 TFLOP/s of fp32 in the products that are computed, bound by the
// matrix instructions: A and A A 0.17-0.18 ms each (253 blocks of 192 x 192, one to a CU), X's update 0.29-0.31 ms.
// 2000 x 1021 bf16 0.29 ms: 21, 14 and 22 us a step; the two squares have 136 blocks of 64 x 64 for 256 CUs, each
// going through its k alone. 4 x 128 x 256 110 us: 17 launches of 6 to 8 us.
//
// Scaling: fp16 holds 2^-24 ... 65504, so each factor is held times a power of two from a bound of its
// entries: |X_k| <= u_k, the largest singular value that the polynomial can reach from at most 1 (found on the
// host), and |X_k| <= f l_k for inputs whose norm eps dwarfs (f = ||G|| / (||G|| + eps)); |A| <= |X|^2 bound. A bound
// sits at 2^14. The norm is summed in fp64.
#include "dense.h"

using namespace dense;
using tile::KIND_SPLIT;

namespace {

constexpr int kMaxSteps = 32;
constexpr int kNormBlocks = 1024;  // partial sums of squares per matrix

// log2 of a step's bounds of the singular values of X, and what the norm makes of the second.
struct Bound {
  float u, l;
};
struct Info {
  float log2_f;
};

__device__ __forceinline__ int exponent(float log2_bound) {
  const float e = 14.0f - ceilf(log2_bound);
  return (int)fminf(fmaxf(e, -100.0f), 120.0f);
}
__device__ __forceinline__ float bound_of(const Bound &b, const Info *info) { return fminf(b.u, info[blockIdx.y].log2_f + b.l); }
__device__ __forceinline__ int x_exponent(float bound) { return exponent(bound); }
__device__ __forceinline__ int a_exponent(float bound) { return exponent(2.0f * bound); }
// |b A + c A A| <= |b| A + |c| A^2, A the bound's square
__device__ __forceinline__ int b_exponent(float bound, float b, float c) {
  const float one = log2f(fabsf(b)) + 2.0f * bound, two = log2f(fabsf(c)) + 4.0f * bound;
  return exponent(fmaxf(one, two) + 1.0f);
}

template <class T>
struct Source {
  const T *data;
  int64_t ld, batch, rows, cols;
};

// The sum over a workgroup of 256, in one order.
__device__ __forceinline__ double sum_of_workgroup(double s, double (&part)[4]) {
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  return part[0] + part[1] + part[2] + part[3];
}

// Sums of squares in fp64, one per workgroup.
template <class T>
__global__ __launch_bounds__(256) void k_squares(Source<T> g, double *parts) {
  __shared__ double part[4];
  const T *m = g.data + blockIdx.y * g.batch;
  double s = 0.0;
  for (int64_t r = blockIdx.x; r < g.rows; r += gridDim.x) {
#pragma unroll 4
    for (int64_t c = threadIdx.x; c < g.cols; c += 256) {
      const double v = load_as_float(m + r * g.ld + c);
      s = fma(v, v, s);
    }
  }
  s = sum_of_workgroup(s, part);
  if (threadIdx.x == 0) parts[blockIdx.y * kNormBlocks + blockIdx.x] = s;
}

__device__ __forceinline__ double sum_of_parts(const double *parts, int count, double (&part)[4]) {
  double s = 0.0;
  for (int i = threadIdx.x; i < count; i += 256) s += parts[blockIdx.y * kNormBlocks + i];
  return sum_of_workgroup(s, part);
}

// The start: X_0 in two parts, and the norm's part of the bounds.
template <class T>
__global__ __launch_bounds__(256) void k_start(Source<T> g, const double *parts, int count, double eps, Bound bound, Info *info, char *x, int64_t pitch) {
  __shared__ double part[4];
  const double norm = sqrt(sum_of_parts(parts, count, part)), inverse = 1.0 / (norm + eps);
  const float log2_f = (float)log2(norm * inverse);
  if (blockIdx.x == 0 && threadIdx.x == 0) info[blockIdx.y].log2_f = log2_f;
  const int e = x_exponent(fminf(bound.u, log2_f + bound.l));
  const T *m = g.data + blockIdx.y * g.batch;
  char *out = x + blockIdx.y * (g.rows * pitch);
  const int64_t wide = pitch / 4;
  for (int64_t r = blockIdx.x; r < g.rows; r += gridDim.x)
    for (int64_t c = threadIdx.x * 4; c < wide; c += 1024) {
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (c + i < g.cols) v[i] = ldexpf((float)(load_as_float(m + r * g.ld + c + i) * inverse), e);
      store_split4(out + r * pitch, c, v);
    }
}

__device__ __forceinline__ f32x4 load_split4(const char *row, int64_t k) {
  const f16x4 hi = *(const f16x4 *)(row + split_at(k)), lo = *(const f16x4 *)(row + split_at(k) + kLow);
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (float)hi[i] + (float)lo[i];
  return v;
}

// The square factor in two parts: A from its sums, or b A + c A A from A A's and A. Blocks off the diagonal are
// written to both sides of it.
struct Square {
  const char *a;  // nullptr: the sums are A
  char *out;
  int64_t size, pitch;
  float b, c;
  Bound bound;
  const Info *info;
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool mirror) const {
    const int lane = threadIdx.x & 63, i16 = lane & 15, j4 = lane >> 4;
    const float limit = bound_of(bound, info);
    const int ex = x_exponent(limit), ea = a_exponent(limit), eb = b_exponent(limit, b, c);
    const int64_t skip = blockIdx.y * (size * pitch);
    char *to = out + skip;
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t m = row0 + 16 * i + i16;
      if (m >= size) continue;
#pragma unroll
      for (int j = 0; j < B::kTN; ++j) {
        const int64_t n = col0 + 16 * j + 4 * j4;
        if (4 * n >= pitch) continue;
        f32x4 v = block.acc[i][j];
        if (a) {
          const f32x4 one = load_split4(a + skip + m * pitch, n);
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = ldexpf(b * ldexpf(one[k], -ea) + c * ldexpf(v[k], -2 * ea), eb);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = ldexpf(v[k], ea - 2 * ex);
        }
        store_split4(to + m * pitch, n, v);
        if (mirror)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (n + k < size) {
              _Float16 hi, lo;
              split(v[k], hi, lo);
              char *p = to + (n + k) * pitch + split_at(m);
              *(_Float16 *)p = hi;
              *(_Float16 *)(p + kLow) = lo;
            }
      }
    }
  }
};

// A from the slabs of a product whose k was split: 4 columns a lane.
__global__ __launch_bounds__(256) void k_square(const float *slabs, int splits, int64_t size, int64_t pitch, char *out, Bound bound, const Info *info) {
  const float limit = bound_of(bound, info);
  const int e = a_exponent(limit) - 2 * x_exponent(limit);
  const int per = (int)(pitch / 16);
  char *to = out + blockIdx.y * (size * pitch);
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < size * per; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per, c = (i - r * per) * 4;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = 0; s < splits; ++s) v += *(const f32x4 *)(slabs + (((int64_t)s * gridDim.y + blockIdx.y) * size + r) * (pitch / 4) + c);
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = ldexpf(v[k], e);
    store_split4(to + r * pitch, c, v);
  }
}

// X's next value, a X + the product's sums: the next factor in two parts, or the answer.
template <class T>
struct Update {
  const char *x;
  char *next;  // nullptr: the last step
  T *out;
  int64_t ld, batch, rows, cols, pitch;
  bool vec;
  float a, b, c;
  Bound bound, after;
  const Info *info;
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
    const int lane = threadIdx.x & 63, i16 = lane & 15, j4 = lane >> 4;
    const float limit = bound_of(bound, info);
    const int ex = x_exponent(limit), eb = b_exponent(limit, b, c), en = x_exponent(bound_of(after, info));
    const int64_t skip = blockIdx.y * (rows * pitch);
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t m = row0 + 16 * i + i16;
      if (m >= rows) continue;
#pragma unroll
      for (int j = 0; j < B::kTN; ++j) {
        const int64_t n = col0 + 16 * j + 4 * j4;
        if (4 * n >= pitch) continue;
        f32x4 v = load_split4(x + skip + m * pitch, n);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = a * ldexpf(v[k], -ex) + ldexpf(block.acc[i][j][k], -ex - eb);
        if (next) {
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = ldexpf(v[k], en);
          store_split4(next + skip + m * pitch, n, v);
        } else if (n < cols) {
          store4(out + blockIdx.y * batch + m * ld + n, v, (int)(cols - n < 4 ? cols - n : 4), vec);
        }
      }
    }
  }
};

// Small matrices: one workgroup does all steps of one matrix, whose X (m x n, m <= n, transposed on the way in and out where
// rows > cols) and square factor stay in LDS in two parts. The launches of the large form cost 17 times 6 us whatever their
// size; here 64 x 64 takes 24 us (105 there), 128 x 128 55 (100), 32 x 1000 54 (105), 1024 of 128 x 128 235 (891).
// 16 waves share the 32 x 32 tiles of each product; every wave computes its tiles into registers, all meet, and the
// tiles are written. LDS holds 32 columns of all rows at a time (a slab), 128 bytes a row as in tile.h, chunks permuted by
// the row; both products' fragments are read from that one form.
constexpr int kRoom = 152 * 1024;
inline int64_t pad32(int64_t x) { return ceil_div(x, 32) * 32; }
inline bool is_small(int64_t rows, int64_t cols) {
  const int64_t m = pad32(std::min(rows, cols)), n = pad32(std::max(rows, cols));
  return m <= 128 && (m * n + m * m) * 4 <= kRoom;  // at most 16 tiles of the square, at most 3 tiles of X a wave
}

struct Steps {
  int count;
  float a, b, c;
  Bound bounds[kMaxSteps + 1];
};
__device__ __forceinline__ float limit_of(const Steps &s, int k, float log2_f) { return fminf(s.bounds[k].u, log2_f + s.bounds[k].l); }

// A 16-row fragment of k = 32 values: part q of rows first ... first + 15 of a slab.
__device__ __forceinline__ tile::i32x4 fragment_along(const char *slab, int first, int q, int lane) {
  const int row = first + (lane & 15);
  return *(const tile::i32x4 *)(slab + row * 128 + (((4 * q + (lane >> 4)) ^ (row & 7)) * 16));
}
// The same of 16 columns (half `half` of the slab's 32) over rows k ... k + 31.
__device__ __forceinline__ tile::i32x4 fragment_across(const char *slab, int k, int half, int q, int lane) {
  typedef __attribute__((address_space(3))) tile::i16x4 lds_i16x4;
  const int r = (lane & 15) >> 2, p = lane & 3, chunk = 4 * q + 2 * half + (p >> 1);
  tile::i16x4 h[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    const int row = k + 8 * (lane >> 4) + 4 * u + r;
    h[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(slab + row * 128 + ((chunk ^ (4 * u + r)) * 16) + (p & 1) * 8));
  }
  return __builtin_bit_cast(tile::i32x4, h);
}

struct Tile32 {
  f32x4 v[2][2];  // [rows 16 i + lane % 16][columns 16 j + 4 (lane / 16)]
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i >> 1][i & 1] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  __device__ __forceinline__ void multiply(const tile::i32x4 (&a)[2][2], const tile::i32x4 (&b)[2][2]) {
#pragma unroll
    for (int part = 2; part >= 0; --part)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) v[i][j] = tile::mfma<KIND_SPLIT>(b[j][part == 1], a[i][part == 2], v[i][j]);
  }
};

// Where part q of four neighbours lies.
__device__ __forceinline__ char *place(char *slab, int row, int col, int q) { return slab + row * 128 + (((4 * q + ((col & 31) >> 3)) ^ (row & 7)) * 16) + (col & 4) * 2; }
__device__ __forceinline__ void put(char *slab, int row, int col, f32x4 v) {
  f16x4 hi, lo;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    _Float16 h, l;
    split(v[i], h, l);
    hi[i] = h;
    lo[i] = l;
  }
  *(f16x4 *)place(slab, row, col, 0) = hi;
  *(f16x4 *)place(slab, row, col, 1) = lo;
}
__device__ __forceinline__ f32x4 get(char *slab, int row, int col) {
  const f16x4 hi = *(const f16x4 *)place(slab, row, col, 0), lo = *(const f16x4 *)place(slab, row, col, 1);
  f32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = (float)hi[i] + (float)lo[i];
  return v;
}

template <class T>
__global__ __launch_bounds__(1024) void k_small(Source<T> g, T *out, int64_t ldo, int64_t batch_o, bool vec, double eps, Steps steps) {
  __shared__ __attribute__((aligned(1024))) char room[kRoom];
  __shared__ double part[16];
  const int tid = threadIdx.x, wave = tile::uniform(tid >> 6);
  int lane = tid & 63;
  const bool tall = g.rows > g.cols;
  const int M = (int)(tall ? g.cols : g.rows), N = (int)(tall ? g.rows : g.cols);
  const int m = (M + 31) & ~31, n = (N + 31) & ~31, slab = m * 128, row_tiles = m / 32, slabs = n / 32;
  char *x = room, *square = room + m * n * 4;
  const T *src = g.data + blockIdx.x * g.batch;
  T *dst = out + blockIdx.x * batch_o;

  // g's values go to LDS as they are, four where their two parts will lie, while their squares are summed. (Lanes
  // go along g's rows; reads outside it are clamped to its last value and dropped, so that all are on their way at once.)
  const int wide = tall ? m : n / 4, items = m * n / 4;
  const auto walk = [&](auto f) {
    int fast = tid % wide, slow = tid / wide;
    const int fast_step = 1024 % wide, slow_step = 1024 / wide;
#pragma unroll 4
    for (int i = tid; i < items; i += 1024) {
      f(tall ? fast : slow, 4 * (tall ? slow : fast));
      fast += fast_step;
      slow += slow_step;
      if (fast >= wide) {
        fast -= wide;
        ++slow;
      }
    }
  };
  double s = 0.0;
  walk([&](int r, int c) {
    f32x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int rr = min(r, M - 1), cc = min(c + k, N - 1);
      const float w = load_as_float(tall ? src + (int64_t)cc * g.ld + rr : src + (int64_t)rr * g.ld + cc);
      v[k] = r < M && c + k < N ? w : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) s = fma((double)v[k], (double)v[k], s);
    char *slab_of = x + (c >> 5) * slab;
    *(float2 *)place(slab_of, r, c, 0) = float2{v[0], v[1]};
    *(float2 *)place(slab_of, r, c, 1) = float2{v[2], v[3]};
  });
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
  if (lane == 0) part[wave] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < 16; ++w) s += part[w];
  const double norm = sqrt(s), inverse = 1.0 / (norm + eps);
  const float log2_f = (float)log2(norm * inverse);
  const int e0 = x_exponent(limit_of(steps, 0, log2_f));
  walk([&](int r, int c) {
    char *slab_of = x + (c >> 5) * slab;
    const float2 one = *(const float2 *)place(slab_of, r, c, 0), two = *(const float2 *)place(slab_of, r, c, 1);
    f32x4 v = {one.x, one.y, two.x, two.y};
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = ldexpf((float)(v[k] * inverse), e0);
    put(slab_of, r, c, v);
  });
  __syncthreads();
  // this wave's tile of the square; for A, as many waves share a tile's k as the room takes their sums
  const int square_tiles = row_tiles * row_tiles, group = wave / square_tiles, tile = wave % square_tiles;
  const int groups = max(1, min(min(16 / square_tiles, slabs / 2), 1 + (kRoom - (m * n + m * m) * 4) / (square_tiles * 4096)));
  f32x4 *sums = (f32x4 *)(square + m * m * 4);
  const int ti = tile / row_tiles, tj = tile % row_tiles;
  const bool squares = group == 0;
  Tile32 next[3];
  for (int step = 0; step < steps.count; ++step) {
    asm volatile("" : "+v"(lane));  // (addresses that do not change are found again each step: kept, they would fill the registers)
    const int i16 = lane & 15, j4 = lane >> 4;
    const float limit = limit_of(steps, step, log2_f);
    const int ex = x_exponent(limit), ea = a_exponent(limit), eb = b_exponent(limit, steps.b, steps.c);
    Tile32 t;
    // A = X X^T
    if (group < groups) {
      t.clear();
#pragma unroll 1
      for (int k = group; k < slabs; k += groups) {
        tile::i32x4 a[2][2], b[2][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i >> 1][i & 1] = fragment_along(x + k * slab, ti * 32 + 16 * (i >> 1), i & 1, lane);
          b[i >> 1][i & 1] = fragment_along(x + k * slab, tj * 32 + 16 * (i >> 1), i & 1, lane);
        }
        t.multiply(a, b);
      }
      if (group > 0)
#pragma unroll
        for (int i = 0; i < 4; ++i) sums[(((group - 1) * square_tiles + tile) * 4 + i) * 64 + lane] = t.v[i >> 1][i & 1];
    }
    if (groups > 1) __syncthreads();
    if (squares) {
      for (int u = 1; u < groups; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) t.v[i >> 1][i & 1] += sums[(((u - 1) * square_tiles + tile) * 4 + i) * 64 + lane];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          f32x4 v = t.v[i][j];
#pragma unroll
          for (int k = 0; k < 4; ++k) v[k] = ldexpf(v[k], ea - 2 * ex);
          put(square + tj * slab, ti * 32 + 16 * i + i16, tj * 32 + 16 * j + 4 * j4, v);
        }
    }
    __syncthreads();
    // b A + c A A
    if (squares) {
      t.clear();
#pragma unroll 1
      for (int k = 0; k < row_tiles; ++k) {
        tile::i32x4 a[2][2], b[2][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i >> 1][i & 1] = fragment_along(square + k * slab, ti * 32 + 16 * (i >> 1), i & 1, lane);
          b[i >> 1][i & 1] = fragment_along(square + k * slab, tj * 32 + 16 * (i >> 1), i & 1, lane);
        }
        t.multiply(a, b);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const f32x4 one = get(square + tj * slab, ti * 32 + 16 * i + i16, tj * 32 + 16 * j + 4 * j4);
#pragma unroll
          for (int k = 0; k < 4; ++k) t.v[i][j][k] = ldexpf(steps.b * ldexpf(one[k], -ea) + steps.c * ldexpf(t.v[i][j][k], -2 * ea), eb);
        }
    }
    __syncthreads();
    if (squares)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) put(square + tj * slab, ti * 32 + 16 * i + i16, tj * 32 + 16 * j + 4 * j4, t.v[i][j]);
    __syncthreads();
    // a X + B X: up to three tiles a wave, held until all have read X
    const bool last = step + 1 == steps.count;
    const int en = last ? 0 : x_exponent(limit_of(steps, step + 1, log2_f)), tiles = row_tiles * slabs;
#pragma unroll
    for (int u = 0; u < 3; ++u) {
      const int id = wave + 16 * u;
      if (id >= tiles) continue;
      const int r = id % row_tiles, c = id / row_tiles;
      next[u].clear();
#pragma unroll 1
      for (int k = 0; k < row_tiles; ++k) {
        tile::i32x4 a[2][2], b[2][2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i >> 1][i & 1] = fragment_along(square + k * slab, r * 32 + 16 * (i >> 1), i & 1, lane);
          b[i >> 1][i & 1] = fragment_across(x + c * slab, k * 32, i >> 1, i & 1, lane);
        }
        next[u].multiply(a, b);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const int row = r * 32 + 16 * i + i16, col = c * 32 + 16 * j + 4 * j4;
          const f32x4 old = get(x + c * slab, row, col);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            next[u].v[i][j][k] = ldexpf(steps.a * ldexpf(old[k], -ex) + ldexpf(next[u].v[i][j][k], -ex - eb), en);
          }
        }
    }
    if (last) break;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 3; ++u) {
      const int id = wave + 16 * u;
      if (id >= tiles) continue;
      const int r = id % row_tiles, c = id / row_tiles;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) put(x + c * slab, r * 32 + 16 * i + i16, c * 32 + 16 * j + 4 * j4, next[u].v[i][j]);
    }
    __syncthreads();
  }
  // the last step's tiles are the answer
  const int i16 = lane & 15, j4 = lane >> 4;
#pragma unroll
  for (int u = 0; u < 3; ++u) {
    const int id = wave + 16 * u;
    if (id >= row_tiles * slabs) continue;
    const int r = id % row_tiles, c = id / row_tiles;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int row = r * 32 + 16 * i + i16, col = c * 32 + 16 * j + 4 * j4;
        if (tall) {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (row < M && col + k < N) dst[(int64_t)(col + k) * ldo + row] = (T)next[u].v[i][j][k];
        } else if (row < M && col < N) {
          store4(dst + row * ldo + col, next[u].v[i][j], min(N - col, 4), vec);
        }
      }
  }
}

// No step: the start itself.
template <class T>
__global__ __launch_bounds__(256) void k_scale(Source<T> g, const double *parts, int count, double eps, T *out, int64_t ld, int64_t batch) {
  __shared__ double part[4];
  const double inverse = 1.0 / (sqrt(sum_of_parts(parts, count, part)) + eps);
  for (int64_t r = blockIdx.x; r < g.rows; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < g.cols; c += 256)
      out[blockIdx.y * batch + r * ld + c] = (T)(float)(load_as_float(g.data + blockIdx.y * g.batch + r * g.ld + c) * inverse);
}

// The largest |p(x)| and |p(x) / x| for x in [0, u], p(x) = a x + b x^3 + c x^5: at u, at 0 or where the derivative is 0.
void reach(double a, double b, double c, double u, double &value, double &slope) {
  const auto p = [&](double s) { return std::fabs(a + b * s + c * s * s); };  // of x^2
  const double s1 = u * u;
  value = u * p(s1);
  slope = std::max(std::fabs(a), p(s1));
  const auto at = [&](double s) {
    if (s > 0.0 && s < s1) {
      value = std::max(value, std::sqrt(s) * p(s));
      slope = std::max(slope, p(s));
    }
  };
  if (c != 0.0) {
    at(-b / (2.0 * c));
    const double d = 9.0 * b * b - 20.0 * a * c;
    if (d >= 0.0) {
      at((-3.0 * b + std::sqrt(d)) / (10.0 * c));
      at((-3.0 * b - std::sqrt(d)) / (10.0 * c));
    }
  } else if (b != 0.0) {
    at(-a / (3.0 * b));
  }
}

struct Space {
  Plan gram, power, update;
  bool split;  // A's k is split: all its blocks are computed, and k_square joins them
  double *parts;
  Info *info;
  char *x[2], *a, *b;
  float *slabs;
  Space(Carver &c, int64_t batch, int64_t rows, int64_t cols) {
    const int64_t m = std::min(rows, cols), k = std::max(rows, cols);
    const bool tall = rows > cols;
    gram = plan(KIND_SPLIT, m, m, k, 1, tall ? kAnyForm : kAlong, batch, true);
    const Plan joined = plan(KIND_SPLIT, m, m, k, kMaxSplits, tall ? kAnyForm : kAlong, batch);
    split = joined.splits > 1 && joined.us < gram.us;
    if (split) gram = joined;
    power = plan(KIND_SPLIT, m, m, m, 1, kAlong, batch, true);
    update = plan(KIND_SPLIT, rows, cols, m, 1, tall ? kAlong : kAnyForm, batch);
    parts = c.take<double>((size_t)(batch * kNormBlocks));
    info = c.take<Info>((size_t)batch);
    for (char *&p : x) p = c.take<char>((size_t)(batch * rows * ceil_div(cols, 32) * 128));
    a = c.take<char>((size_t)(batch * m * ceil_div(m, 32) * 128));
    b = c.take<char>((size_t)(batch * m * ceil_div(m, 32) * 128));
    slabs = c.take<float>(split ? (size_t)(gram.splits * batch * m * ceil_div(m, 32) * 32) : 0);
  }
};

template <class T>
sdnn_status orthogonalize(const T *g, int64_t ldg, int64_t batch_g, T *out, int64_t ldo, int64_t batch_o, int64_t batch, int64_t rows, int64_t cols, int steps, const float *coef, float eps,
                          void *workspace, hipStream_t stream) {
  Carver carver{(char *)workspace};
  const Space sp(carver, batch, rows, cols);
  const Source<T> src{g, ldg, batch_g, rows, cols};
  Steps plan_of{steps, coef[0], coef[1], coef[2], {}};
  Bound *bounds = plan_of.bounds;
  double u = 1.0, l = 1.0;
  for (int k = 0; k <= steps; ++k) {
    bounds[k] = {(float)std::log2(u), (float)std::log2(l)};
    double value, slope;
    reach(coef[0], coef[1], coef[2], u, value, slope);
    u = std::min(1e30, std::max(1e-30, 1.01 * value));  // what rounding adds is far below a hundredth
    l = std::min(1e30, std::max(1e-30, 1.01 * slope * l));
  }
  const bool vec = (uintptr_t)out % (4 * sizeof(T)) == 0 && ldo % 4 == 0 && batch_o % 4 == 0;
  if (steps > 0 && is_small(rows, cols)) {
    hipLaunchKernelGGL((k_small<T>), dim3((unsigned)batch), dim3(1024), 0, stream, src, out, ldo, batch_o, vec, (double)eps, plan_of);
    return launched("orthogonalize");
  }
  const unsigned norm_blocks = (unsigned)std::min<int64_t>(rows, kNormBlocks), row_blocks = (unsigned)std::min<int64_t>(rows, 2048);
  hipLaunchKernelGGL((k_squares<T>), dim3(norm_blocks, (unsigned)batch), dim3(256), 0, stream, src, sp.parts);
  if (steps == 0) {
    hipLaunchKernelGGL((k_scale<T>), dim3(row_blocks, (unsigned)batch), dim3(256), 0, stream, src, sp.parts, (int)norm_blocks, (double)eps, out, ldo, batch_o);
    return launched("orthogonalize");
  }
  const int64_t pitch = ceil_div(cols, 32) * 128, m = std::min(rows, cols), square = ceil_div(m, 32) * 128;
  hipLaunchKernelGGL((k_start<T>), dim3(row_blocks, (unsigned)batch), dim3(256), 0, stream, src, sp.parts, (int)norm_blocks, (double)eps, bounds[0], sp.info, sp.x[0], pitch);
  sdnn_status st = launched("orthogonalize");
  const bool tall = rows > cols;
  for (int k = 0; k < steps && st == SDNN_OK; ++k) {
    const char *x = sp.x[k & 1];
    char *next = k + 1 < steps ? sp.x[(k + 1) & 1] : nullptr;
    const Matrix mx{x, pitch, rows, pitch, rows * pitch}, ma{sp.a, square, m, square, m * square}, mb{sp.b, square, m, square, m * square};
    Square e{nullptr, sp.a, m, square, coef[1], coef[2], bounds[k], sp.info};
    if (sp.split) {
      const Accumulate parts{sp.slabs, square / 4, m, m, false};
      st = tall ? run_shape<KIND_SPLIT, true, true>(sp.gram, mx, mx, m, m, rows, parts, stream, "orthogonalize", false, (int)batch)
                : run_shape<KIND_SPLIT, false, false>(sp.gram, mx, mx, m, m, cols, parts, stream, "orthogonalize", false, (int)batch);
      if (st != SDNN_OK) return st;
      hipLaunchKernelGGL(k_square, dim3((unsigned)std::min<int64_t>(ceil_div(m * (square / 16), 256), 2048), (unsigned)batch), dim3(256), 0, stream, sp.slabs, sp.gram.splits, m, square, sp.a, bounds[k],
                         sp.info);
      st = launched("orthogonalize");
    } else {
      st = tall ? run_shape<KIND_SPLIT, true, true>(sp.gram, mx, mx, m, m, rows, e, stream, "orthogonalize", true, (int)batch)
                : run_shape<KIND_SPLIT, false, false>(sp.gram, mx, mx, m, m, cols, e, stream, "orthogonalize", true, (int)batch);
    }
    if (st != SDNN_OK) return st;
    e.a = sp.a;
    e.out = sp.b;
    st = run_shape<KIND_SPLIT, false, false>(sp.power, ma, ma, m, m, m, e, stream, "orthogonalize", true, (int)batch);
    if (st != SDNN_OK) return st;
    const Update<T> last{x, next, out, ldo, batch_o, rows, cols, pitch, vec, coef[0], coef[1], coef[2], bounds[k], bounds[k + 1], sp.info};
    st = tall ? run_shape<KIND_SPLIT, false, false>(sp.update, mx, mb, rows, cols, m, last, stream, "orthogonalize", false, (int)batch)
              : run_shape<KIND_SPLIT, false, true>(sp.update, mb, mx, rows, cols, m, last, stream, "orthogonalize", false, (int)batch);
  }
  return st;
}

}  // namespace

extern "C" {

size_t sdnn_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols) {
  if (batch < 0 || batch > 65535 || rows < 1 || rows > kMaxFeatures || cols < 1 || cols > kMaxFeatures) return 0;
  Carver c{nullptr};
  Space s(c, batch, rows, cols);
  return c.used;
}

sdnn_status sdnn_orthogonalize(const void *g, int64_t ldg, int64_t batch_stride_g, void *out, int64_t ldo, int64_t batch_stride_o, int32_t dtype, int64_t batch, int64_t rows, int64_t cols,
                               int32_t steps, const float *coefficients, float eps, void *workspace, size_t workspace_bytes, void *hip_stream) {
  if (batch < 0 || batch > 65535) return fail(SDNN_EINVAL, "batch %lld is outside [0, 65535]", (long long)batch);
  if (rows < 1 || rows > kMaxFeatures) return fail(SDNN_EINVAL, "rows %lld is outside [1, %lld]", (long long)rows, (long long)kMaxFeatures);
  if (cols < 1 || cols > kMaxFeatures) return fail(SDNN_EINVAL, "cols %lld is outside [1, %lld]", (long long)cols, (long long)kMaxFeatures);
  if (!good_dtype(dtype)) return fail(SDNN_EINVAL, "dtype %d is neither SDNN_FP32 nor SDNN_BF16", dtype);
  if (steps < 0 || steps > kMaxSteps) return fail(SDNN_EINVAL, "steps %d is outside [0, %d]", steps, kMaxSteps);
  if (!coefficients) return fail(SDNN_EINVAL, "coefficients is null");
  for (int i = 0; i < 3; ++i)
    if (!(std::fabs(coefficients[i]) <= 1e6f)) return fail(SDNN_EINVAL, "coefficient %d is not in [-1e6, 1e6]", i);
  if (!(eps >= 0.0f && eps <= 1e30f)) return fail(SDNN_EINVAL, "eps is not in [0, 1e30]");
  if (batch == 0) return SDNN_OK;
  sdnn_status st;
  if ((st = check_matrix("g", g, ldg, cols, dtype)) != SDNN_OK) return st;
  if ((st = check_matrix("out", out, ldo, cols, dtype)) != SDNN_OK) return st;
  if (batch > 1 && (batch_stride_g < 0 || batch_stride_g > (1ll << 40) || batch_stride_o < (rows - 1) * ldo + cols || batch_stride_o > (1ll << 40)))
    return fail(SDNN_EINVAL, "a batch stride is out of range");
  if ((st = check_workspace(workspace, workspace_bytes, sdnn_orthogonalize_workspace_bytes(batch, rows, cols))) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (dtype == SDNN_BF16)
    return orthogonalize((const __bf16 *)g, ldg, batch_stride_g, (__bf16 *)out, ldo, batch_stride_o, batch, rows, cols, steps, coefficients, eps, workspace, stream);
  return orthogonalize((const float *)g, ldg, batch_stride_g, (float *)out, ldo, batch_stride_o, batch, rows, cols, steps, coefficients, eps, workspace, stream);
}

}  // extern "C"
