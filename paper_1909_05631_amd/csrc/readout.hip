// The dense readout of a network's rows: softmax cross entropy of l = x w^T (n_rows x n_classes) and its gradient,
// in pieces of the classes and without keeping l.
//
//   lse_t = log sum_v exp l_tv,  loss_t = lse_t - l_{t, y_t}
//   G_tv = g_t (exp(l_tv - lse_t) - [v = y_t]),  dx = G w,  dw = G^T x
//
// A row whose label is outside [0, n_classes) is left out: loss 0, gradient 0, and nothing of it reaches dw,
// whatever it holds.
//
// Loss: one pass over w. A block of up to 256 rows by as many classes has its logits in registers; the epilogue takes
// the maximum and the sum of exponentials of its columns per row (fp32), k_loss joins them: 8 bytes are written for 32 to
// 64 logits. Past 2^30 logits rows and classes are gone over in panels of that many, a row's softmax so far is carried
// from one panel of its classes to the next, and what is written grows no more. Where there are few logits (at most
// 2^24) and blocks for only a part of the CUs, the features are split instead, and a workgroup a row joins the slabs
// and takes the softmax.
// Gradient: piece by piece, the logits are computed again (2 of 8 T V D operations, against a logit matrix in memory),
// the epilogue writes the piece's G (bf16; fp32 inputs: three bf16 parts), and two products read it, dx +=
// G w (over the piece's classes) and dw = G^T x (over the rows), both through the transposing LDS reads, so neither
// w, x nor G is ever transposed in memory. A piece holds at most 2^26 values of G (or 256 classes of all rows): in bf16
// it stays in the Infinity Cache between the products.
//
// What bounds it, measured on this card (a copy runs at 4.8 TB/s, the library's bf16 product at 1650 TFLOP/s once the
// clock has settled under load, 1290 in its first passes; fp16 1555):
//   8192 x 4096 x 32768, bf16: 6.5 ms, matrix instructions: loss 1.59 ms (1386 TFLOP/s), each of four pieces
//     0.42-0.43 ms logits and G, 0.40-0.42 ms dx, 0.36-0.37 ms dw (1470-1520).
//   64 x 1024 x 65536, bf16: 136 us, memory: w three times (23-25 us each, 5.4-5.8 TB/s), dw once (35 us, 3.8 TB/s).
//   1021 x 1000 x 10007, fp32: 451 us: logits 62 us in the loss (333 TFLOP/s of fp32 in two fp16 parts, of 518) and 85 us
//     with G's three parts stored; dx 98 us, dw 133 us (209 and 154 TFLOP/s in three bf16 parts, of 275; dw has
//     160 blocks for 256 CUs); 64 us for writing x and w in parts, once a call.
//   2000 x 1024 x 10, fp32: 45 us, eight launches of 5 to 8 us.
//
// fp32 inputs go to the logits as two fp16 parts under a power of two per row of x and of w, which the logits' own
// rows and columns take back. The gradient's products cannot: their sums run over the rows of x or the classes, whose
// sizes may lie any number of powers of two apart, and one row of x or of w far larger than the others would leave
// these no bits. So G, w and x go there as three bf16 parts, which need no common scale. Where rows or classes are at
// most 192, all go to the fp32 matrix instructions as they are (16 x 1024 x 65536: loss 55 us, 224 with w in two parts).
// One to four rows or classes (few.h) mostly have no use for tiles: one kernel with fp32 arithmetic streams the other
// matrix past them, once.
#include "dense.h"
#include "few.h"

#include <type_traits>

using namespace dense;
using tile::KIND_BF16;
using tile::KIND_F32;
using tile::KIND_SPLIT;
using tile::KIND_THREE;

namespace {

constexpr int64_t kPieceValues = 1 << 26;  // of G at a time
constexpr int64_t kPieceClasses = 1 << 19;
constexpr int64_t kPanel = 1 << 30, kPanelClasses = 1 << 16;  // of logits at a time in the loss, of classes where rows go in panels too
constexpr int64_t kPlain = 192;            // fp32 rows or classes for the plain fp32 products: see Sizes::kind
constexpr int64_t kSplitLogits = 1 << 24;  // logits whose features may be split: past that there is a 256 x 256 block for every CU
constexpr float kLog2e = 1.44269504088896340736f;

// exp, by the hardware's exponential of base 2 (one rounding of the argument, which is at most 0 in the sums: the
// terms that matter have arguments near 0).
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

__device__ __forceinline__ bool counted(const int64_t *labels, int64_t t, int64_t classes) {
  return (uint64_t)labels[t] < (uint64_t)classes;
}

// What the kernels of one call hand on in device memory.
struct Scalars {
  float mean;      // 1 / (number of counted rows), at most 1
  float heaviest;  // the largest magnitude of the counted rows' weights (1 if that is 0)
};

__device__ __forceinline__ float finite_magnitude(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : 0.0f;  // false for NaN too
}

__device__ __forceinline__ float max_of_workgroup(float m, float (&part)[4]) {
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
  __syncthreads();
  return fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3]));
}

// The number of counted rows and their heaviest weight, by a workgroup of 256.
__device__ __forceinline__ void count_rows(const int64_t *labels, int64_t rows, int64_t classes, const float *weights, Scalars *out) {
  __shared__ int part[4];
  __shared__ float tops[4];
  int n = 0;
  float top = 0.0f;
#pragma unroll 8
  for (int64_t t = threadIdx.x; t < rows; t += 256) {
    const bool live = counted(labels, t, classes);
    n += live;
    if (weights && live) top = fmaxf(top, finite_magnitude(weights[t]));
  }
  if (weights) top = max_of_workgroup(top, tops);
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = part[0] + part[1] + part[2] + part[3];
    out->mean = 1.0f / (float)(n > 1 ? n : 1);
    out->heaviest = top > 0.0f ? top : 1.0f;
  }
}
__global__ __launch_bounds__(256) void k_count(const int64_t *labels, int64_t rows, int64_t classes, Scalars *out) { count_rows(labels, rows, classes, nullptr, out); }

__device__ __forceinline__ float top4(f32x4 v) {
  return fmaxf(fmaxf(finite_magnitude(v[0]), finite_magnitude(v[1])), fmaxf(finite_magnitude(v[2]), finite_magnitude(v[3])));
}

// An fp32 matrix's rows for the kernel that goes over x and w in one launch. Rows without a label (labels != nullptr)
// become zeros.
struct Rows {
  const float *data;
  int64_t ld, rows;
  const int64_t *labels;
  int *exponents;  // of each row in two parts
  char *out;       // in two parts, 32 * groups values a row
  char *three;     // in three parts, whole groups of 64 (nullptr: not wanted)
  bool vec;        // rows are 16-byte aligned
};

// fp32 rows in their parts, zeros past `cols`: `first` workgroups on x, the rest on w. With `scalars`, the last
// workgroup counts the rows that have a label.
__global__ __launch_bounds__(256) void k_split_rows(Rows x, Rows w, int first, int64_t cols, int64_t groups, const int64_t *labels, int64_t classes, Scalars *scalars) {
  __shared__ float part[4];
  const int work = (int)gridDim.x - (scalars ? 1 : 0), b = blockIdx.x;
  if (b == work) return count_rows(labels, x.rows, classes, nullptr, scalars);
  const Rows &m = b < first ? x : w;
  const int64_t pitch3 = ceil_div(cols, 64) * tile::kGroup3, wide = m.three ? pitch3 / 6 : groups * 32;
  for (int64_t r = b < first ? b : b - first; r < m.rows; r += b < first ? first : work - first) {
    const float *row = m.data + r * m.ld;
    const bool live = !m.labels || counted(m.labels, r, classes);
    float top = 0.0f;
    if (live)
      for (int64_t k = threadIdx.x * 4; k < cols; k += 1024) top = fmaxf(top, top4(few::load4(row, (int)k, (int)cols, m.vec)));
    const int e = split_exponent(max_of_workgroup(top, part));
    if (threadIdx.x == 0) m.exponents[r] = e;
    char *to = m.out + r * groups * 128;
#pragma unroll 2
    for (int64_t k = threadIdx.x * 4; k < wide; k += 1024) {
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
      if (live) v = few::load4(row, (int)k, (int)cols, m.vec);
      if (m.three) store_three4(m.three + r * pitch3, k, v);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = ldexpf(v[i], e);
      if (k < groups * 32) store_split4(to, k, v);
    }
  }
}

// Rows on 16-byte aligned rows of `pitch` values, zeros past `cols` and in rows without a label. With `scalars`, the last
// workgroup counts the rows that have one and finds the heaviest weight.
template <class T>
__global__ __launch_bounds__(256) void k_copy_rows(const T *x, int64_t ld, int64_t rows, int64_t cols, int64_t pitch, const int64_t *labels, int64_t classes, const float *weights, bool vec, T *out,
                                                   Scalars *scalars) {
  if (scalars && blockIdx.x == gridDim.x - 1) return count_rows(labels, rows, classes, weights, scalars);
  constexpr int kEach = 16 / sizeof(T);
  typedef T Chunk __attribute__((ext_vector_type(kEach)));
  const int step = (int)gridDim.x - (scalars ? 1 : 0);
  for (int64_t r = blockIdx.x; r < rows; r += step) {
    const bool live = !labels || counted(labels, r, classes);
    for (int64_t k = threadIdx.x * kEach; k < pitch; k += 256 * kEach) {
      Chunk v = {};
      if (live) {
        if (vec && k + kEach <= cols) {
          v = *(const Chunk *)(x + r * ld + k);
        } else {
#pragma unroll
          for (int i = 0; i < kEach; ++i)
            if (k + i < cols) v[i] = x[r * ld + k + i];
        }
      }
      *(Chunk *)(out + r * pitch + k) = v;
    }
  }
}

// What turns a block's sums into logits: the exponents of the operands' rows and columns (split).
struct LogitScale {
  const int *row, *col;
};

// Loss: per row and the wave's columns, the largest logit and the sum of exponentials against it.
template <int KIND>
struct LossParts {
  LogitScale scale;
  const int64_t *labels;
  int64_t rows, first, classes;  // of the panel; its first class
  float2 *parts;   // [rows][count]
  int64_t count;   // parts of a row
  float *picked;   // the label's logit
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
    const int lane = threadIdx.x & 63, i16 = lane & 15, j4 = lane >> 4;
    constexpr int kWide = 16 * B::kTN;
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t t = row0 + 16 * i + i16;
      const bool in = t < rows;
      const int er = KIND == KIND_SPLIT && in ? scale.row[t] : 0;
      const int64_t y = in ? labels[t] - first : -1;
      float l[4 * B::kTN], m = -__builtin_inff();
#pragma unroll
      for (int j = 0; j < B::kTN; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const int64_t v = col0 + 16 * j + 4 * j4 + c;
          float s = block.acc[i][j][c];
          if (KIND == KIND_SPLIT) s = ldexpf(s, -er - (v < classes ? scale.col[v] : 0));
          if (in && v == y) picked[t] = s;
          if (v >= classes) s = -__builtin_inff();
          l[4 * j + c] = s;
          m = fmaxf(m, s);
        }
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      float sum = 0.0f;
#pragma unroll
      for (int k = 0; k < 4 * B::kTN; ++k) sum += l[k] == -__builtin_inff() ? 0.0f : exp_of(l[k] - m);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      if (in && j4 == 0 && col0 < classes) parts[t * count + col0 / kWide] = float2{m, sum};
    }
  }
};

// Joins the parts of a row, and what is carried of the panels before: one wave a row, or a workgroup where there are many. A NaN logit makes NaN of its row's
// sum (the maximum passes it over).
struct Softmax {
  float top, sum;
  __device__ __forceinline__ void join(float t, float s) {
    const float n = fmaxf(top, t);
    sum = (top == -__builtin_inff() ? sum : sum * exp_of(top - n)) + (t == -__builtin_inff() ? s : s * exp_of(t - n));
    top = n;
  }
};
// The rows of a panel and what their softmax comes to.
struct Losses {
  const float *picked;
  const int64_t *labels;
  int64_t rows, classes;  // all classes
  float *loss, *lse;
  float2 *carried;   // nullptr: all classes are in one panel
  bool first, last;  // of the panels of these rows' classes
};
template <int WAVES>
__global__ __launch_bounds__(256) void k_loss(const float2 *parts, int64_t count, Losses to) {
  __shared__ float2 shared[4];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t = WAVES == 1 ? (int64_t)blockIdx.x * 4 + wave : blockIdx.x;
  if (WAVES == 1 && t >= to.rows) return;
  Softmax a{-__builtin_inff(), 0.0f};
#pragma unroll 4
  for (int64_t p = threadIdx.x & (64 * WAVES - 1); p < count; p += 64 * WAVES) {
    const float2 b = parts[t * count + p];
    a.join(b.x, b.y);
  }
  for (int d = 32; d; d >>= 1) {
    const float top = __shfl_xor(a.top, d), sum = __shfl_xor(a.sum, d);
    a.join(top, sum);
  }
  if constexpr (WAVES > 1) {
    if (lane == 0) shared[wave] = float2{a.top, a.sum};
    __syncthreads();
    a = {shared[0].x, shared[0].y};
    for (int w = 1; w < 4; ++w) a.join(shared[w].x, shared[w].y);
  }
  if (lane == 0 && (WAVES == 1 || wave == 0)) {
    if (!to.first) a.join(to.carried[t].x, to.carried[t].y);
    if (!to.last) {
      to.carried[t] = float2{a.top, a.sum};
      return;
    }
    const float s = a.top + logf(a.sum);
    if (to.lse) to.lse[t] = s;
    to.loss[t] = counted(to.labels, t, to.classes) ? s - to.picked[t] : 0.0f;
  }
}

// The loss from logits whose k was split: a workgroup sums a row's slabs and takes its softmax.
template <int KIND>
__global__ __launch_bounds__(256) void k_loss_slabs(const float *slabs, int splits, int64_t ld, LogitScale scale, const int64_t *labels, int64_t rows, int64_t classes, float *loss, float *lse) {
  __shared__ float2 shared[4];
  __shared__ float picked;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const int64_t t = blockIdx.x, y = labels[t];
  Softmax a{-__builtin_inff(), 0.0f};
  for (int64_t v = threadIdx.x; v < classes; v += 256) {
    float l = 0.0f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) l += slabs[(s * rows + t) * ld + v];
    if (KIND == KIND_SPLIT) l = ldexpf(l, -scale.row[t] - scale.col[v]);
    if (v == y) picked = l;
    a.join(l, l == -__builtin_inff() ? 0.0f : 1.0f);
  }
  for (int d = 32; d; d >>= 1) {
    const float top = __shfl_xor(a.top, d), sum = __shfl_xor(a.sum, d);
    a.join(top, sum);
  }
  if (lane == 0) shared[wave] = float2{a.top, a.sum};
  __syncthreads();
  if (threadIdx.x == 0) {
    a = {shared[0].x, shared[0].y};
    for (int w = 1; w < 4; ++w) a.join(shared[w].x, shared[w].y);
    const float s = a.top + logf(a.sum);
    if (lse) lse[t] = s;
    loss[t] = counted(labels, t, classes) ? s - picked : 0.0f;
  }
}

sdnn_status join_parts(const float2 *parts, int64_t count, const Losses &to, hipStream_t stream) {
  if (count > 256 && to.rows < 8 * kCus)
    hipLaunchKernelGGL((k_loss<4>), dim3((unsigned)to.rows), dim3(256), 0, stream, parts, count, to);
  else
    hipLaunchKernelGGL((k_loss<1>), dim3((unsigned)ceil_div(to.rows, 4)), dim3(256), 0, stream, parts, count, to);
  return launched("loss");
}

// Gradient: the piece's exp(l - lse) - [v = y], zeros in rows without a label, times the row's weight. Three parts of
// fp32: as that is. Else: over the heaviest weight, so that equal weights (a mean's) are a factor of one and, in bf16,
// the label's -1 is exact; a common factor that were rounded here would be off by as much in every row's gradient.
template <int KIND>
struct WriteGrad {
  LogitScale scale;  // the piece's columns
  const int64_t *labels;
  const float *lse, *weights;
  const Scalars *scalars;
  int64_t rows, all, first, classes;  // all classes; the piece's first and number
  char *g;
  int64_t pitch;  // bytes
  __device__ __forceinline__ float heaviest() const { return KIND != KIND_SPLIT && weights ? scalars->heaviest : 1.0f; }
  // What a row's values have in common.
  struct Row {
    bool live;
    int64_t y;
    float z, w;
    int e;
  };
  __device__ __forceinline__ Row row(int64_t t, bool in, float heaviest) const {
    const bool live = in && counted(labels, t, all);
    return {live, in ? labels[t] - first : -1, live ? lse[t] : 0.0f, weights && live ? weights[t] / heaviest : 1.0f, KIND == KIND_SPLIT && in ? scale.row[t] : 0};
  }
  // Four neighbours of a row, from class v of the piece on.
  __device__ __forceinline__ f32x4 gradient(f32x4 l, int64_t v, const Row &r) const {
    f32x4 o;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
      const bool in = v + c < classes;
      const float s = KIND == KIND_SPLIT ? ldexpf(l[c], -r.e - (in ? scale.col[v + c] : 0)) : l[c];
      const float p = exp_of(s - r.z) - (v + c == r.y ? 1.0f : 0.0f);
      o[c] = r.live && in ? r.w * p : 0.0f;
    }
    return o;
  }
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
    const int lane = threadIdx.x & 63, i16 = lane & 15, j4 = lane >> 4;
    const float heavy = heaviest();
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t t = row0 + 16 * i + i16;
      const bool in = t < rows;
      const Row r = row(t, in, heavy);
      const auto value = [&](int j) { return gradient(block.acc[i][j], col0 + 16 * j + 4 * j4, r); };
      if constexpr (KIND == KIND_SPLIT) {
#pragma unroll
        for (int j = 0; j < B::kTN; ++j) {
          const int64_t v = col0 + 16 * j + 4 * j4;
          const f32x4 o = value(j);
          if (in && v < pitch / 6) store_three4(g + t * pitch, v, o);
        }
      } else {
        using G = std::conditional_t<KIND == KIND_F32, float, __bf16>;
        store_row<G, B::kTN>((G *)(g + t * pitch), col0, pitch / (int)sizeof(G), true, in, value);
      }
    }
  }
};

// The same from logits whose k was split.
template <int KIND>
__global__ __launch_bounds__(256) void k_grad_slabs(const float *slabs, int splits, int64_t ld, WriteGrad<KIND> to) {
  const int64_t t = blockIdx.y;
  const typename WriteGrad<KIND>::Row r = to.row(t, true, to.heaviest());
  char *row = to.g + t * to.pitch;
  const int64_t wide = to.pitch / (KIND == KIND_BF16 ? 2 : KIND == KIND_SPLIT ? 6 : 4);
  for (int64_t v = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; v < wide; v += (int64_t)gridDim.x * 1024) {
    f32x4 l = {0.0f, 0.0f, 0.0f, 0.0f};
    if (v < ld)
#pragma unroll 4
      for (int s = 0; s < splits; ++s) l += *(const f32x4 *)(slabs + (s * to.rows + t) * ld + v);
    const f32x4 o = to.gradient(l, v, r);
    if constexpr (KIND == KIND_SPLIT)
      store_three4(row, v, o);
    else if constexpr (KIND == KIND_F32)
      store4((float *)row + v, o, 4, true);
    else
      store4((__bf16 *)row + v, o, 4, true);
  }
}

template <class T>
struct Store {
  T *out;
  int64_t ld, rows, cols;
  bool vec;
  const float *factor = nullptr;  // what the sums are multiplied by: the mean's, or the heaviest weight
  const float *before = nullptr;  // sums of the pieces before
  int64_t ld_before = 0;
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
    const int i16 = threadIdx.x & 15;
    const float by = factor ? *factor : 1.0f;
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t r = row0 + 16 * i + i16;
      const bool in = r < rows;
      store_row<T, B::kTN>(out + r * ld, col0, cols, vec, in, [&](int j) {
        f32x4 v = block.acc[i][j];
        const int64_t c = col0 + 16 * j + 4 * ((threadIdx.x & 63) >> 4);
        if (before && in && c < ld_before) v += *(const f32x4 *)(before + r * ld_before + c);
        return v * by;
      });
    }
  }
};

// The slabs' sum, rounded to the output's type: 256 / GROUPS items a workgroup, each group taking every GROUPS-th slab.
template <class T, int GROUPS>
__global__ __launch_bounds__(256) void k_sum_slabs(const float *slabs, int splits, int64_t ld_slab, Store<T> to) {
  constexpr int kItems = 256 / GROUPS;
  __shared__ f32x4 shared[GROUPS][kItems];
  const int64_t per = ld_slab / 4, total = to.rows * per;
  const float by = to.factor ? *to.factor : 1.0f;
  const int group = threadIdx.x / kItems, item = threadIdx.x % kItems;
  for (int64_t i0 = (int64_t)blockIdx.x * kItems; i0 < total; i0 += (int64_t)gridDim.x * kItems) {
    const int64_t i = i0 + item, r = i / per, c = (i - r * per) * 4;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i < total)
#pragma unroll 8
      for (int s = group; s < splits; s += GROUPS) v += *(const f32x4 *)(slabs + (s * to.rows + r) * ld_slab + c);
    if constexpr (GROUPS > 1) {
      __syncthreads();
      shared[group][item] = v;
      __syncthreads();
      if (group == 0)
        for (int g = 1; g < GROUPS; ++g) v += shared[g][item];
    }
    if (group == 0 && i < total && c < to.cols) store4(to.out + r * to.ld + c, v * by, (int)(to.cols - c < 4 ? to.cols - c : 4), to.vec);
  }
}

template <class T>
sdnn_status sum_slabs(const float *slabs, int splits, int64_t ld_slab, const Store<T> &to, hipStream_t stream, const char *what) {
  const int64_t items = to.rows * (ld_slab / 4);
  if (splits >= 32)
    hipLaunchKernelGGL((k_sum_slabs<T, 16>), dim3((unsigned)std::min<int64_t>(ceil_div(items, 16), 8192)), dim3(256), 0, stream, slabs, splits, ld_slab, to);
  else if (splits >= 8)
    hipLaunchKernelGGL((k_sum_slabs<T, 4>), dim3((unsigned)std::min<int64_t>(ceil_div(items, 64), 8192)), dim3(256), 0, stream, slabs, splits, ld_slab, to);
  else
    hipLaunchKernelGGL((k_sum_slabs<T, 1>), dim3((unsigned)std::min<int64_t>(ceil_div(items, 256), 8192)), dim3(256), 0, stream, slabs, splits, ld_slab, to);
  return launched(what);
}

// ------------------------------------------------------------------------------------------------
// Host

constexpr int kWaveCols[kShapes] = {64, 48, 48, 64, 64, 32, 32, 32, 32};  // columns of a wave: the parts of a row of logits

// The size of equal parts of `all`, of at most about `most` each and whole units but for the last.
int64_t part_of(int64_t all, int64_t most, int64_t unit) { return std::min(all, ceil_div(ceil_div(all, ceil_div(all, most)), unit) * unit); }

// Sizes of one call.
struct Sizes {
  int64_t rows, classes, features;
  int32_t dtype;
  int64_t per_slab() const { return dtype == SDNN_BF16 ? 64 : 32; }
  int64_t groups() const { return ceil_div(features, 32); }
  int64_t pitch_values() const { return ceil_div(features, 8) * 8; }  // rows that had to be copied
  size_t three(int64_t n) const { return (size_t)(n * three_pitch()); }
  int64_t three_pitch() const { return ceil_div(features, 64) * tile::kGroup3; }
  size_t packed(int64_t n) const { return kind() == KIND_SPLIT ? (size_t)(n * groups() * 128) : (size_t)(n * pitch_values() * dtype_bytes(dtype)); }
  // fp32 operands go to the fp32 matrix instructions as they are up to kPlain rows or classes: the other matrix is
  // then the larger one, and writing it in parts costs more than faster products save. Loss and gradient, us, as they are
  // and in parts: 64 x 1024 x 65536 374 and 794; 160 rows 833 and 972; 192 rows 856 and 984; 256 rows 1160 and 1045; 512
  // rows 2259 and 1524; 192 x 1000 x 10007 173 both, 256 rows 223 and 196; 60000 x 1024 x 130 classes 928 and 949, 200
  // classes 1211 and 1019. (Small products gain by it past that, 512 x 512 x 512 66 and 70, 5000 x 200 x 256 65 and 81.)
  int kind() const { return dtype == SDNN_BF16 ? KIND_BF16 : std::min(rows, classes) <= kPlain ? KIND_F32 : KIND_SPLIT; }
  // The loss's panels: all of it, or equal parts of whole blocks (256 rows, 256 or 192 classes): a last one of a few
  // classes would be a launch that fills few CUs (60000 x 1024 x 65536 bf16: 7.5 ms, 7.8 with last panels of 256 classes; 7.3
  // in one launch, whose parts take twice the memory).
  int64_t panel_classes() const { return rows * classes <= kPanel ? classes : part_of(classes, std::max(kPanelClasses, kPanel / rows), 768); }
  int64_t panel_rows() const { return rows * classes <= kPanel ? rows : part_of(rows, std::max<int64_t>(256, kPanel / panel_classes() / 256 * 256), 256); }
  // Classes of a piece: 2^26 values of G, whole blocks of 256 classes.
  int64_t piece() const {
    const int64_t p = std::max<int64_t>(256, std::min(kPieceClasses, kPieceValues / std::max<int64_t>(rows, 1)) / 256 * 256);
    return std::min(p, classes);
  }
  int64_t g_pitch() const { return kind() == KIND_SPLIT ? ceil_div(piece(), 64) * tile::kGroup3 : ceil_div(piece(), per_slab()) * 128; }
  // The logits' k may be split where they are few: their slabs are joined by a row's workgroup (5 x 5000 x 1000 fp32: loss
  // 21 us, 102 unsplit; gradient 42 and 127; 2100 x 2100 x 8192 bf16: 83 and 283, unsplit 125 and 331;
  // 500 x 12000 x 4096 bf16: 72 us either way).
  int logit_splits(int64_t n) const { return rows * n <= kSplitLogits && rows <= 65535 ? kMaxSplits : 1; }
  Plan logits(int64_t n) const { return plan(kind(), rows, n, features, logit_splits(n), kAlong); }
  size_t logit_slabs(const Plan &p, int64_t n) const { return p.splits > 1 ? (size_t)(p.splits * rows * (ceil_div(n, 4) * 4)) : 0; }
  int product_kind() const { return kind() == KIND_SPLIT ? KIND_THREE : kind(); }
  Plan dx() const { return plan(product_kind(), rows, features, piece(), kMaxSplits); }
  Plan dw(int64_t n) const { return plan(product_kind(), n, features, rows, kMaxSplits); }
  int64_t ld_slab() const { return ceil_div(features, 4) * 4; }
  few::Fit fit(bool rows_held) const { return rows_held ? few::fit_of(rows, classes, features, dtype) : few::fit_of(classes, rows, features, dtype); }
  // Few rows are held rather than few classes.
  bool rows_held() const { return fit(true) != few::kNone && (rows <= classes || fit(false) == few::kNone); }
  few::Fit few() const { return fit(rows_held()); }
};

// Rows that the tiles read as they are: whole dwords.
bool usable_in_place(const void *p, int64_t ld, int64_t cols, int bytes) {
  return ((uintptr_t)p & 3) == 0 && ld * bytes % 4 == 0 && cols * bytes % 4 == 0 && ld * bytes <= kMaxPitch;
}

// A call's workspace and the plans of its products.
struct LossSpace {
  Plan loss{};
  char *x, *w;
  int *ex, *ew;
  float2 *parts, *carried;
  float *picked, *slabs;
  int64_t count;
  LossSpace(Carver &c, const Sizes &s) {
    const bool packed = s.few() == few::kNone;
    if (packed) loss = s.logits(s.classes);
    x = c.take<char>(packed ? s.packed(s.rows) : 0);
    w = c.take<char>(packed ? s.packed(s.classes) : 0);
    ex = c.take<int>(s.rows);
    ew = c.take<int>(s.classes);
    count = !packed ? (s.rows_held() ? (int64_t)few::grid_of(s.few(), s.classes, false) * few::batch_of(s.few()) : 0) : ceil_div(s.panel_classes(), kWaveCols[loss.shape]);
    parts = c.take<float2>((packed ? s.panel_rows() : s.rows) * count);
    carried = c.take<float2>(packed && s.panel_classes() < s.classes ? s.panel_rows() : 0);
    picked = c.take<float>(s.rows);
    slabs = c.take<float>(packed ? s.logit_slabs(loss, s.classes) : 0);
  }
};

struct GradSpace {
  Plan logits, dx_plan, dw_plan[2];  // dw: of a whole piece and of the last one
  char *x, *w, *x3, *w3, *g;
  int *ex, *ew;
  Scalars *scalars;
  float *dx, *dw, *few, *slabs;
  GradSpace(Carver &c, const Sizes &s) {
    scalars = c.take<Scalars>(1);
    if (s.few() != ::few::kNone) {
      const bool held = s.rows_held();
      few = c.take<float>((size_t)(::few::grid_of(s.few(), held ? s.classes : s.rows, true) * (held ? s.rows : s.classes) * s.ld_slab()));
      return;
    }
    x = c.take<char>(s.packed(s.rows));
    w = c.take<char>(s.packed(s.classes));
    const bool split = s.kind() == KIND_SPLIT;
    x3 = c.take<char>(split ? s.three(s.rows) : 0);
    w3 = c.take<char>(split ? s.three(s.classes) : 0);
    ex = c.take<int>(split ? s.rows : 0);
    ew = c.take<int>(split ? s.classes : 0);
    g = c.take<char>((size_t)(s.rows * s.g_pitch()));
    const int64_t piece = s.piece(), rest = s.classes % piece;
    dx_plan = s.dx();
    dx = c.take<float>(dx_plan.splits > 1 || piece < s.classes ? (size_t)(dx_plan.splits * s.rows * s.ld_slab()) : 0);
    // the loss's blocks and parts of k, whatever the piece: the logits are those that lse was taken of, to the bit. With
    // sums in another order a logit of 1e6 would be off by a sixteenth against its own lse, and a certain answer not certain.
    logits = s.logits(s.classes);
    size_t most = 0;
    for (int i = 0; i < 2; ++i) {
      const int64_t n = i == 0 ? piece : rest;
      if (n == 0) continue;
      dw_plan[i] = s.dw(n);
      if (dw_plan[i].splits > 1) most = std::max(most, (size_t)(dw_plan[i].splits * n * s.ld_slab()));
    }
    dw = c.take<float>(most);
    slabs = c.take<float>(s.logit_slabs(logits, piece));
  }
};

unsigned row_grid(int64_t rows) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(rows, 2048)); }

bool aligned16(const void *p, int64_t ld, int bytes) { return ((uintptr_t)p & 15) == 0 && ld * bytes % 16 == 0; }

// Rows as an operand of their own type: in place, or copied into `space` (always with labels; then the counted rows are
// counted too).
template <class T>
Matrix plain_rows(const T *data, int64_t ld, int64_t rows, const Sizes &s, const int64_t *labels, const float *weights, Scalars *scalars, char *space, hipStream_t stream) {
  constexpr int kBytes = sizeof(T);
  if (!labels && usable_in_place(data, ld, s.features, kBytes)) return {(const char *)data, ld * kBytes, rows, s.features * kBytes, 0};
  hipLaunchKernelGGL((k_copy_rows<T>), dim3(row_grid(rows) + (scalars ? 1 : 0)), dim3(256), 0, stream, data, ld, rows, s.features, s.pitch_values(), labels, s.classes, weights,
                     aligned16(data, ld, kBytes), (T *)space, scalars);
  return {space, s.pitch_values() * kBytes, rows, s.pitch_values() * kBytes, 0};
}

Matrix split_matrix(const Rows &r, const Sizes &s) { return {r.out, s.groups() * 128, r.rows, s.groups() * 128, 0}; }

Matrix three_matrix(const Rows &r, const Sizes &s) { return {r.three, s.three_pitch(), r.rows, ceil_div(s.features, 8) * 16, 0}; }

// x and w in their parts; with `scalars` the rows that have a label are counted too.
void split_rows(const Rows &x, const Rows &w, const Sizes &s, const int64_t *labels, Scalars *scalars, hipStream_t stream) {
  const unsigned a = row_grid(x.rows), b = row_grid(w.rows);
  hipLaunchKernelGGL(k_split_rows, dim3(a + b + (scalars ? 1 : 0)), dim3(256), 0, stream, x, w, (int)a, s.features, s.groups(), labels, s.classes, scalars);
}

template <class T>
bool vector_rows(const T *p, int64_t ld) {  // aligned for 16 bytes
  return (uintptr_t)p % 16 == 0 && ld * sizeof(T) % 16 == 0;
}

template <class T>
few::Few<T> few_of(const Sizes &s, const T *x, int64_t ldx, const T *w, int64_t ldw, const int64_t *labels) {
  const bool rows = s.rows_held();
  few::Few<T> p{};
  p.held = rows ? x : w;
  p.stream = rows ? w : x;
  p.ld_held = rows ? ldx : ldw;
  p.ld_stream = rows ? ldw : ldx;
  p.held_rows = (int)(rows ? s.rows : s.classes);
  p.stream_rows = rows ? s.classes : s.rows;
  p.features = (int)s.features;
  p.vec_held = s.features % 4 == 0 && vector_rows(p.held, p.ld_held);
  p.vec_stream = s.features % 4 == 0 && vector_rows(p.stream, p.ld_stream);
  p.labels = labels;
  p.classes = s.classes;
  return p;
}

template <int KIND, class T>
sdnn_status loss_of(const Sizes &s, const T *x, int64_t ldx, const T *w, int64_t ldw, const int64_t *labels, float *loss, float *lse, void *workspace, size_t workspace_bytes,
                    hipStream_t stream) {
  Carver carver{(char *)workspace};
  const LossSpace sp(carver, s);
  sdnn_status st = check_workspace(workspace, workspace_bytes, carver.used);
  if (st != SDNN_OK) return st;
  if (s.few() != few::kNone) {
    few::Few<T> p = few_of(s, x, ldx, w, ldw, labels);
    p.loss = loss;
    p.lse = lse;
    p.parts = sp.parts;
    p.picked = sp.picked;
    if (!s.rows_held()) return few::launch<false, false>(s.few(), p, stream, "loss");
    st = few::launch<true, false>(s.few(), p, stream, "loss");
    return st != SDNN_OK ? st : join_parts(sp.parts, sp.count, Losses{sp.picked, labels, s.rows, s.classes, loss, lse, nullptr, true, true}, stream);
  }
  Matrix a, b;
  if constexpr (KIND != KIND_SPLIT) {
    a = plain_rows(x, ldx, s.rows, s, nullptr, nullptr, nullptr, sp.x, stream);
    b = plain_rows(w, ldw, s.classes, s, nullptr, nullptr, nullptr, sp.w, stream);
  } else {
    const Rows rx{x, ldx, s.rows, nullptr, sp.ex, sp.x, nullptr, aligned16(x, ldx, 4)};
    const Rows rw{w, ldw, s.classes, nullptr, sp.ew, sp.w, nullptr, aligned16(w, ldw, 4)};
    split_rows(rx, rw, s, labels, nullptr, stream);
    a = split_matrix(rx, s);
    b = split_matrix(rw, s);
  }
  if ((st = launched("rows")) != SDNN_OK) return st;
  const LogitScale scale{sp.ex, sp.ew};
  if (sp.loss.splits > 1) {
    const int64_t ld = ceil_div(s.classes, 4) * 4;
    st = run_shape<KIND, false, false>(sp.loss, a, b, s.rows, s.classes, s.features, Accumulate{sp.slabs, ld, s.rows, s.classes, false}, stream, "loss");
    if (st != SDNN_OK) return st;
    hipLaunchKernelGGL((k_loss_slabs<KIND>), dim3((unsigned)s.rows), dim3(256), 0, stream, sp.slabs, sp.loss.splits, ld, scale, labels, s.rows, s.classes, loss, lse);
    return launched("loss");
  }
  const int64_t panel = s.panel_rows(), piece = s.panel_classes();
  for (int64_t t0 = 0; t0 < s.rows; t0 += panel)
    for (int64_t v0 = 0; v0 < s.classes; v0 += piece) {
      const int64_t m = std::min(panel, s.rows - t0), n = std::min(piece, s.classes - v0);
      Matrix ap = a, bp = b;
      ap.data += t0 * a.pitch;
      bp.data += v0 * b.pitch;
      ap.rows = m;
      bp.rows = n;
      const int64_t count = ceil_div(n, kWaveCols[sp.loss.shape]);
      const LossParts<KIND> e{{sp.ex + t0, sp.ew + v0}, labels + t0, m, v0, n, sp.parts, count, sp.picked + t0};
      st = run_shape<KIND, false, false>(sp.loss, ap, bp, m, n, s.features, e, stream, "loss");
      if (st != SDNN_OK) return st;
      const Losses to{sp.picked + t0, labels + t0, m, s.classes, loss + t0, lse ? lse + t0 : nullptr, sp.carried, v0 == 0, v0 + n == s.classes};
      st = join_parts(sp.parts, count, to, stream);
      if (st != SDNN_OK) return st;
    }
  return SDNN_OK;
}

// C = A B^T over k, into `to` directly or through fp32 slabs.
template <int KIND, bool AA, class T>
sdnn_status product(const Plan &p, const Matrix &a, const Matrix &b, int64_t k, float *slabs, int64_t ld_slab, bool through, bool add, bool last, const Store<T> &to, hipStream_t stream, const char *what) {
  if (!through) return run_shape<KIND, AA, true>(p, a, b, to.rows, to.cols, k, to, stream, what);
  const Accumulate e{slabs, ld_slab, to.rows, to.cols, add};
  sdnn_status st = run_shape<KIND, AA, true>(p, a, b, to.rows, to.cols, k, e, stream, what);
  if (st != SDNN_OK || !last) return st;
  return sum_slabs(slabs, p.splits, ld_slab, to, stream, what);
}

template <class T>
__global__ __launch_bounds__(256) void k_zero_rows(T *out, int64_t ld, int64_t rows, int64_t cols) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < cols; c += 256) out[r * ld + c] = (T)0.0f;
}

template <int KIND, class T>
sdnn_status grad_of(const Sizes &s, const T *x, int64_t ldx, const T *w, int64_t ldw, const int64_t *labels, const float *lse, const float *weights, T *dx, int64_t lddx, T *dw, int64_t lddw,
                    void *workspace, size_t workspace_bytes, hipStream_t stream) {
  Carver carver{(char *)workspace};
  const GradSpace sp(carver, s);
  sdnn_status st = check_workspace(workspace, workspace_bytes, carver.used);
  if (st != SDNN_OK) return st;
  if (s.rows == 0) {
    if (dw) hipLaunchKernelGGL((k_zero_rows<T>), dim3(row_grid(s.classes)), dim3(256), 0, stream, dw, lddw, s.classes, s.features);
    return launched("gradient");
  }
  if (s.few() != few::kNone) {
    const bool held = s.rows_held();
    few::Few<T> p = few_of(s, x, ldx, w, ldw, labels);
    T *d_held = held ? dx : dw;
    const int64_t ld_d_held = held ? lddx : lddw;
    p.known_lse = lse;
    p.weights = weights;
    p.mean = &sp.scalars->mean;
    p.d_stream = held ? dw : dx;
    p.ld_d = held ? lddw : lddx;
    p.vec_d = vector_rows(p.d_stream, p.ld_d);
    p.slabs = d_held ? sp.few : nullptr;
    p.ld_slab = s.ld_slab();
    if (!held && !weights) hipLaunchKernelGGL(k_count, dim3(1), dim3(256), 0, stream, labels, s.rows, s.classes, sp.scalars);
    st = held ? few::launch<true, true>(s.few(), p, stream, "gradient") : few::launch<false, true>(s.few(), p, stream, "gradient");
    if (st != SDNN_OK || !d_held) return st;
    const Store<T> to{d_held, ld_d_held, p.held_rows, s.features, vector_rows(d_held, ld_d_held)};
    return sum_slabs(sp.few, (int)few::grid_of(s.few(), p.stream_rows, true), s.ld_slab(), to, stream, "gradient");
  }
  constexpr int kProduct = KIND == KIND_SPLIT ? KIND_THREE : KIND;
  Matrix a, b, ag, bg;  // ag, bg: the rows of x and w as dw's and dx's products take them
  if constexpr (KIND != KIND_SPLIT) {
    ag = a = plain_rows(x, ldx, s.rows, s, labels, weights, sp.scalars, sp.x, stream);
    bg = b = plain_rows(w, ldw, s.classes, s, nullptr, nullptr, nullptr, sp.w, stream);
  } else {
    const Rows rx{x, ldx, s.rows, labels, sp.ex, sp.x, dw ? sp.x3 : nullptr, aligned16(x, ldx, 4)};
    const Rows rw{w, ldw, s.classes, nullptr, sp.ew, sp.w, dx ? sp.w3 : nullptr, aligned16(w, ldw, 4)};
    split_rows(rx, rw, s, labels, sp.scalars, stream);
    a = split_matrix(rx, s);
    b = split_matrix(rw, s);
    ag = three_matrix(rx, s);
    bg = three_matrix(rw, s);
  }
  st = launched("gradient");
  // what the products are multiplied by in the end: the mean's factor, or the weights'
  const float *factor = !weights ? &sp.scalars->mean : KIND != KIND_SPLIT ? &sp.scalars->heaviest : nullptr;
  const Plan &px = sp.dx_plan;
  const int64_t piece = s.piece();
  const bool through_x = px.splits > 1 || piece < s.classes;
  for (int64_t v0 = 0; v0 < s.classes && st == SDNN_OK; v0 += piece) {
    const int64_t n = std::min(piece, s.classes - v0);
    const bool last = v0 + n == s.classes;
    Matrix wp = b, wg = bg;  // the piece's classes
    wp.data += v0 * b.pitch;
    wg.data += v0 * bg.pitch;
    wp.rows = wg.rows = n;
    const WriteGrad<KIND> e{{sp.ex, sp.ew + v0}, labels, lse, weights, sp.scalars, s.rows, s.classes, v0, n, sp.g, s.g_pitch()};
    const Plan &pl = sp.logits;
    if (pl.splits > 1) {
      const int64_t ld = ceil_div(n, 4) * 4;
      st = run_shape<KIND, false, false>(pl, a, wp, s.rows, n, s.features, Accumulate{sp.slabs, ld, s.rows, n, false}, stream, "gradient");
      if (st != SDNN_OK) return st;
      hipLaunchKernelGGL((k_grad_slabs<KIND>), dim3((unsigned)std::min<int64_t>(ceil_div(s.g_pitch(), 2048), 64), (unsigned)s.rows), dim3(256), 0, stream, sp.slabs, pl.splits, ld, e);
      st = launched("gradient");
    } else {
      st = run_shape<KIND, false, false>(pl, a, wp, s.rows, n, s.features, e, stream, "gradient");
    }
    if (st != SDNN_OK) return st;
    const int64_t wide = ceil_div(n * (int64_t)(kProduct == KIND_THREE ? 2 : sizeof(T)), 16) * 16;  // bytes of a row of G (of one part)
    if (dx) {
      const Store<T> to{dx, lddx, s.rows, s.features, vector_rows(dx, lddx), factor, v0 > 0 && px.splits == 1 ? sp.dx : nullptr, s.ld_slab()};
      const bool direct = !through_x || (last && px.splits == 1);
      st = product<kProduct, false>(px, Matrix{sp.g, s.g_pitch(), s.rows, wide, 0}, wg, n, sp.dx, s.ld_slab(), !direct, v0 > 0, last, to, stream, "gradient of the rows");
      if (st != SDNN_OK) return st;
    }
    if (dw) {
      const Plan &pw = sp.dw_plan[n < piece];
      const Store<T> to{dw + v0 * lddw, lddw, n, s.features, vector_rows(dw + v0 * lddw, lddw), factor};
      st = product<kProduct, true>(pw, Matrix{sp.g, s.g_pitch(), s.rows, wide, 0}, ag, s.rows, sp.dw, s.ld_slab(), pw.splits > 1, false, true, to, stream, "gradient of the weights");
    }
  }
  return st;
}

sdnn_status check_sizes(int64_t n_rows, int64_t n_classes, int64_t n_features, int32_t dtype) {
  if (n_rows < 0 || n_rows > kMaxRows) return fail(SDNN_EINVAL, "n_rows %lld is outside [0, %lld]", (long long)n_rows, (long long)kMaxRows);
  if (n_classes < 1 || n_classes > kMaxClasses) return fail(SDNN_EINVAL, "n_classes %lld is outside [1, %lld]", (long long)n_classes, (long long)kMaxClasses);
  if (n_features < 1 || n_features > kMaxFeatures) return fail(SDNN_EINVAL, "n_features %lld is outside [1, %lld]", (long long)n_features, (long long)kMaxFeatures);
  if (!good_dtype(dtype)) return fail(SDNN_EINVAL, "dtype %d is neither SDNN_FP32 nor SDNN_BF16", dtype);
  return SDNN_OK;
}

}  // namespace

extern "C" {

size_t sdnn_readout_workspace_bytes(int64_t n_rows, int64_t n_classes, int64_t n_features, int32_t dtype, int32_t gradient) {
  if (check_sizes(n_rows, n_classes, n_features, dtype) != SDNN_OK) return 0;
  const Sizes s{n_rows, n_classes, n_features, dtype};
  Carver loss{nullptr}, grad{nullptr};
  LossSpace a(loss, s);
  if (!gradient) return loss.used;
  GradSpace b(grad, s);
  return std::max(loss.used, grad.used);
}

sdnn_status sdnn_readout_loss(const void *x, int64_t ldx, const void *w, int64_t ldw, int32_t dtype, const int64_t *labels, int64_t n_rows, int64_t n_classes, int64_t n_features, float *loss,
                              float *lse, void *workspace, size_t workspace_bytes, void *hip_stream) {
  sdnn_status st = check_sizes(n_rows, n_classes, n_features, dtype);
  if (st != SDNN_OK || n_rows == 0) return st;
  if ((st = check_matrix("x", x, ldx, n_features, dtype)) != SDNN_OK) return st;
  if ((st = check_matrix("w", w, ldw, n_features, dtype)) != SDNN_OK) return st;
  if (!labels || !loss) return fail(SDNN_EINVAL, "labels or loss is null");
  const Sizes s{n_rows, n_classes, n_features, dtype};
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (dtype == SDNN_BF16) return loss_of<KIND_BF16>(s, (const __bf16 *)x, ldx, (const __bf16 *)w, ldw, labels, loss, lse, workspace, workspace_bytes, stream);
  if (s.kind() == KIND_F32) return loss_of<KIND_F32>(s, (const float *)x, ldx, (const float *)w, ldw, labels, loss, lse, workspace, workspace_bytes, stream);
  return loss_of<KIND_SPLIT>(s, (const float *)x, ldx, (const float *)w, ldw, labels, loss, lse, workspace, workspace_bytes, stream);
}

sdnn_status sdnn_readout_grad(const void *x, int64_t ldx, const void *w, int64_t ldw, int32_t dtype, const int64_t *labels, const float *lse, const float *row_grad, int64_t n_rows,
                              int64_t n_classes, int64_t n_features, void *dx, int64_t lddx, void *dw, int64_t lddw, void *workspace, size_t workspace_bytes, void *hip_stream) {
  sdnn_status st = check_sizes(n_rows, n_classes, n_features, dtype);
  if (st != SDNN_OK) return st;
  if (n_rows > 0) {
    if ((st = check_matrix("x", x, ldx, n_features, dtype)) != SDNN_OK) return st;
    if ((st = check_matrix("w", w, ldw, n_features, dtype)) != SDNN_OK) return st;
    if (!labels || !lse) return fail(SDNN_EINVAL, "labels or lse is null");
    if (dx && (st = check_matrix("dx", dx, lddx, n_features, dtype)) != SDNN_OK) return st;
  }
  if (dw && (st = check_matrix("dw", dw, lddw, n_features, dtype)) != SDNN_OK) return st;
  if ((!dx || n_rows == 0) && !dw) return SDNN_OK;
  const Sizes s{n_rows, n_classes, n_features, dtype};
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (dtype == SDNN_BF16)
    return grad_of<KIND_BF16, __bf16>(s, (const __bf16 *)x, ldx, (const __bf16 *)w, ldw, labels, lse, row_grad, (__bf16 *)dx, lddx, (__bf16 *)dw, lddw, workspace, workspace_bytes, stream);
  if (s.kind() == KIND_F32)
    return grad_of<KIND_F32, float>(s, (const float *)x, ldx, (const float *)w, ldw, labels, lse, row_grad, (float *)dx, lddx, (float *)dw, lddw, workspace, workspace_bytes, stream);
  return grad_of<KIND_SPLIT, float>(s, (const float *)x, ldx, (const float *)w, ldw, labels, lse, row_grad, (float *)dx, lddx, (float *)dw, lddw, workspace, workspace_bytes, stream);
}

}  // extern "C"
