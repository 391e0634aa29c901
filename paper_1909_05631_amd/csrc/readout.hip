// The dense readout of a network's rows: softmax cross entropy of l = x w^T (n_rows x n_classes) and its gradient,
// in pieces of the classes and without keeping l.
//
//   lse_t = log sum_v exp l_tv,  loss_t = lse_t - l_{t, y_t}
//   G_tv = g_t (exp(l_tv - lse_t) - [v = y_t]),  dx = G w,  dw = G^T x
//
// A row whose label is outside [0, n_classes) is left out: loss 0, gradient 0, and nothing of it reaches dw,
// whatever it holds.
//
// Loss: one pass over w. A block of 64 ... 256 rows by as many classes has its logits in registers; the epilogue takes
// the maximum and the sum of exponentials of its columns per row (fp32), k_loss joins them. Nothing of size
// n_rows x n_classes is written.
// Gradient: piece by piece, the logits are computed again (2 of 8 T V D operations, against a logit matrix in memory),
// the epilogue writes the piece's G in 16 bits (bf16; fp32 inputs: two fp16 parts), and two products read it, dx +=
// G w (over the piece's classes) and dw = G^T x (over the rows), both through the transposing LDS reads, so neither
// w, x nor G is ever transposed in memory. A piece holds at most 2^26 values of G: it stays in the Infinity Cache
// between the products.
#include "dense.h"

using namespace dense;
using tile::Block;
using tile::KIND_BF16;
using tile::KIND_SPLIT;

namespace {

constexpr int64_t kPieceValues = 1 << 26;  // of G at a time
constexpr int64_t kPieceClasses = 1 << 19;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kTopBlocks = 512;
constexpr int kGradExponent = 15;  // fp16 parts of exp(l - lse) - [v = y] hold it times 2^15

// exp, by the hardware's exponential of base 2 (one rounding of the argument, which is at most 0 in the sums: the
// terms that matter have arguments near 0).
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

__device__ __forceinline__ bool counted(const int64_t *labels, int64_t t, int64_t classes) {
  return (uint64_t)labels[t] < (uint64_t)classes;
}

// What the kernels of one call hand on in device memory.
struct Scalars {
  float top[3][kTopBlocks];  // largest finite magnitudes of x (counted rows), of w, of x times its rows' weights, by workgroup
  float mean;                // 1 / (number of counted rows), at most 1
};

// One workgroup: the number of counted rows.
__global__ __launch_bounds__(1024) void k_count(const int64_t *labels, int64_t rows, int64_t classes, Scalars *out) {
  __shared__ int part[16];
  int n = 0;
  for (int64_t t = threadIdx.x; t < rows; t += 1024) n += counted(labels, t, classes);
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x == 0) {
    n = 0;
    for (int i = 0; i < 16; ++i) n += part[i];
    out->mean = 1.0f / (float)(n > 1 ? n : 1);
  }
}

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

// Largest finite magnitudes of a matrix, of its rows times their weights if there are any: one per workgroup. Rows without a label are skipped.
__global__ __launch_bounds__(256) void k_top(const float *x, int64_t ld, int64_t rows, int64_t cols, const int64_t *labels, int64_t classes, const float *weights, float *top) {
  __shared__ float part[4];
  float m = 0.0f;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    if (labels && !counted(labels, r, classes)) continue;
    const float w = weights ? weights[r] : 1.0f;
#pragma unroll 4
    for (int64_t c = threadIdx.x; c < cols; c += 256) m = fmaxf(m, finite_magnitude(x[r * ld + c] * w));
  }
  m = max_of_workgroup(m, part);
  if (threadIdx.x == 0) top[blockIdx.x] = m;
}

// What k_top found, by one wave (all of its lanes get it).
__device__ __forceinline__ float top_of(const float *top) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < kTopBlocks / 64; ++i) m = fmaxf(m, top[i * 64 + (threadIdx.x & 63)]);
  for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
  return m;
}

// fp32 rows in the split form, 32 * groups values each, zeros past `cols`. A row's exponent: from its own largest
// magnitude (exponents != nullptr, where it is written), or from the whole matrix's (top). weights: the values are
// multiplied by their row's weight first. Rows without a label become zeros.
__global__ __launch_bounds__(256) void k_split_rows(const float *x, int64_t ld, int64_t rows, int64_t cols, int64_t groups, const int64_t *labels, int64_t classes, const float *weights,
                                                    const float *top, int *exponents, char *out) {
  __shared__ float part[4];
  const int whole = exponents ? 0 : split_exponent(top_of(top));
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const float *row = x + r * ld;
    const bool live = !labels || counted(labels, r, classes);
    const float w = weights && live ? weights[r] : 1.0f;
    int e;
    if (exponents) {
      float m = 0.0f;
      if (live)
        for (int64_t c = threadIdx.x; c < cols; c += 256) m = fmaxf(m, finite_magnitude(row[c]));
      e = split_exponent(max_of_workgroup(m, part));
      if (threadIdx.x == 0) exponents[r] = e;
    } else {
      e = whole;
    }
    char *to = out + r * groups * 128;
    for (int64_t k = threadIdx.x * 4; k < groups * 32; k += 1024) {
      f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
      if (live)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (k + i < cols) v[i] = ldexpf(row[k + i] * w, e);
      store_split4(to, k, v);
    }
  }
}

// bf16 rows on 16-byte aligned rows of `pitch` values, zeros past `cols` and in rows without a label.
__global__ __launch_bounds__(256) void k_copy_rows(const __bf16 *x, int64_t ld, int64_t rows, int64_t cols, int64_t pitch, const int64_t *labels, int64_t classes, bool vec, __bf16 *out) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    const bool live = !labels || counted(labels, r, classes);
    for (int64_t k = threadIdx.x * 8; k < pitch; k += 2048) {
      typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
      bf16x8 v = {};
      if (live) {
        if (vec && k + 8 <= cols) {
          v = *(const bf16x8 *)(x + r * ld + k);
        } else {
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (k + i < cols) v[i] = x[r * ld + k + i];
        }
      }
      *(bf16x8 *)(out + r * pitch + k) = v;
    }
  }
}

// What turns a block's sums into logits: the operands' powers of two.
struct LogitScale {
  const int *row, *col;            // exponents by row and column (split, loss)
  const float *top_x, *top_w;      // or of the whole matrices (split, gradient)
};
template <int KIND>
__device__ __forceinline__ int whole_exponent(const LogitScale &s) {
  if (KIND == KIND_BF16 || s.row) return 0;
  return split_exponent(top_of(s.top_x)) + split_exponent(top_of(s.top_w));
}

// Loss: per row and the wave's columns, the largest logit and the sum of exponentials against it.
template <int KIND>
struct LossParts {
  LogitScale scale;
  const int64_t *labels;
  int64_t rows, classes;
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
      const int64_t y = in ? labels[t] : -1;
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

// One wave per row: joins the parts. A NaN logit makes NaN of its row's sum (the maximum passes it over).
__global__ __launch_bounds__(256) void k_loss(const float2 *parts, int64_t count, const float *picked, const int64_t *labels, int64_t rows, int64_t classes, float *loss, float *lse) {
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (t >= rows) return;
  float m = -__builtin_inff(), sum = 0.0f;
  for (int64_t p = lane; p < count; p += 64) {
    const float2 a = parts[t * count + p];
    const float n = fmaxf(m, a.x);
    const float keep = m == -__builtin_inff() ? 0.0f : exp_of(m - n);
    sum = sum * keep + (a.x == -__builtin_inff() ? a.y : a.y * exp_of(a.x - n));
    m = n;
  }
  for (int d = 32; d; d >>= 1) {
    const float om = __shfl_xor(m, d), os = __shfl_xor(sum, d);
    const float n = fmaxf(m, om);
    sum = (m == -__builtin_inff() ? sum : sum * exp_of(m - n)) + (om == -__builtin_inff() ? os : os * exp_of(om - n));
    m = n;
  }
  if (lane == 0) {
    const float s = m + logf(sum);
    if (lse) lse[t] = s;
    loss[t] = counted(labels, t, classes) ? s - picked[t] : 0.0f;
  }
}

// Gradient: the piece's G. bf16: with the row's weight; split: without it, times 2^15.
template <int KIND>
struct WriteGrad {
  LogitScale scale;
  const int64_t *labels;
  const float *lse, *weights;  // weights == nullptr: the mean over the counted rows
  const Scalars *scalars;
  int64_t rows, all, first, classes;  // all classes; the piece's first and number
  char *g;
  int64_t pitch;  // bytes
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
    const int lane = threadIdx.x & 63, i16 = lane & 15, j4 = lane >> 4;
    const int e = whole_exponent<KIND>(scale);
    const float mean = weights ? 0.0f : scalars->mean;
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t t = row0 + 16 * i + i16;
      if (t >= rows) continue;
      const int64_t y = labels[t] - first;
      const bool live = counted(labels, t, all);
      const float z = live ? lse[t] : 0.0f;
      float w = live ? (weights ? weights[t] : mean) : 0.0f;
      if (KIND == KIND_SPLIT) w = 1 << kGradExponent;
#pragma unroll
      for (int j = 0; j < B::kTN; ++j) {
        const int64_t v = col0 + 16 * j + 4 * j4;
        f32x4 o;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          float s = block.acc[i][j][c];
          if (KIND == KIND_SPLIT) s = ldexpf(s, -e);
          const float p = exp_of(s - z) - (v + c == y ? 1.0f : 0.0f);
          o[c] = live && v + c < classes ? w * p : 0.0f;
        }
        if constexpr (KIND == KIND_SPLIT) {
          if (split_at(v) < pitch) store_split4(g + t * pitch, v, o);
        } else {
          if (2 * v < pitch) store4((__bf16 *)(g + t * pitch) + v, o, 4, true);
        }
      }
    }
  }
};

// What a product's sums are multiplied by: the mean and the split operands' powers of two (found once a wave), and
// the row's weight. A sum of zero stays zero whatever the weight: rows without a label.
struct OutScale {
  const float *rows;
  const float *mean;
  const float *top;  // of the operand that was split (nullptr: none)
  struct Found {
    float mean;
    int e;
  };
  __device__ __forceinline__ Found find() const { return {mean ? *mean : 1.0f, top ? -kGradExponent - split_exponent(top_of(top)) : 0}; }
  __device__ __forceinline__ float weight(int64_t row) const { return rows ? rows[row] : 1.0f; }
  __device__ __forceinline__ f32x4 apply(Found f, float weight, f32x4 v) const {
#pragma unroll
    for (int k = 0; k < 4; ++k) v[k] = v[k] == 0.0f ? 0.0f : ldexpf(v[k], f.e) * f.mean * weight;
    return v;
  }
};

template <class T>
struct Store {
  T *out;
  int64_t ld, rows, cols;
  bool vec;
  OutScale scale;
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
    const int lane = threadIdx.x & 63, i16 = lane & 15, j4 = lane >> 4;
    const OutScale::Found found = scale.find();
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t r = row0 + 16 * i + i16;
      if (r >= rows) continue;
      const float w = scale.weight(r);
#pragma unroll
      for (int j = 0; j < B::kTN; ++j) {
        const int64_t c = col0 + 16 * j + 4 * j4;
        if (c >= cols) continue;
        store4(out + r * ld + c, scale.apply(found, w, block.acc[i][j]), (int)(cols - c < 4 ? cols - c : 4), vec);
      }
    }
  }
};

// Sums kept in fp32, one slab per part of k; with `add`, on what the pieces before left there.
struct Accumulate {
  float *slabs;
  int64_t ld, rows, cols;
  bool add;
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int split, bool) const {
    const int lane = threadIdx.x & 63, i16 = lane & 15, j4 = lane >> 4;
    float *slab = slabs + split * rows * ld;
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t r = row0 + 16 * i + i16;
      if (r >= rows) continue;
#pragma unroll
      for (int j = 0; j < B::kTN; ++j) {
        const int64_t c = col0 + 16 * j + 4 * j4;
        if (c >= ld) continue;
        f32x4 *p = (f32x4 *)(slab + r * ld + c);
        *p = add ? *p + block.acc[i][j] : block.acc[i][j];
      }
    }
  }
};

// The slabs' sum, in their order, rounded to the output's type.
template <class T>
__global__ __launch_bounds__(256) void k_sum_slabs(const float *slabs, int splits, int64_t ld_slab, Store<T> to) {
  const int64_t per = ld_slab / 4;
  const OutScale::Found found = to.scale.find();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < to.rows * per; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / per, c = (i - r * per) * 4;
    if (c >= to.cols) continue;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = 0; s < splits; ++s) v += *(const f32x4 *)(slabs + (s * to.rows + r) * ld_slab + c);
    store4(to.out + r * to.ld + c, to.scale.apply(found, to.scale.weight(r), v), (int)(to.cols - c < 4 ? to.cols - c : 4), to.vec);
  }
}

// ------------------------------------------------------------------------------------------------
// Host

constexpr int kWaveCols[kShapes] = {64, 48, 64, 32, 32, 32};  // columns of a wave: the parts of a row of logits

// Sizes of one call.
struct Sizes {
  int64_t rows, classes, features;
  int32_t dtype;
  int64_t per_slab() const { return dtype == SDNN_BF16 ? 64 : 32; }
  int64_t groups() const { return ceil_div(features, 32); }
  int64_t pitch_values() const { return ceil_div(features, 8) * 8; }  // bf16 rows that had to be copied
  size_t packed(int64_t n) const { return dtype == SDNN_BF16 ? (size_t)(n * pitch_values() * 2) : (size_t)(n * groups() * 128); }
  int64_t feature_slabs() const { return ceil_div(features, per_slab()); }
  // Classes of a piece: 2^26 values of G, whole blocks of 256 classes.
  int64_t piece() const {
    const int64_t p = std::max<int64_t>(256, std::min(kPieceClasses, kPieceValues / std::max<int64_t>(rows, 1)) / 256 * 256);
    return std::min(p, classes);
  }
  int64_t g_pitch() const { return ceil_div(piece(), per_slab()) * 128; }
  Plan loss() const { return plan(rows, classes, feature_slabs(), 1, kAlong); }
  Plan logits(int64_t n) const { return plan(rows, n, feature_slabs(), 1, kAlong); }
  Plan dx() const { return plan(rows, features, ceil_div(piece(), per_slab()), kMaxSplits); }
  Plan dw(int64_t n) const { return plan(n, features, ceil_div(rows, per_slab()), kMaxSplits); }
  int64_t ld_slab() const { return ceil_div(features, 4) * 4; }
};

bool usable_in_place(const void *p, int64_t ld, int64_t cols) {
  return ((uintptr_t)p & 15) == 0 && ld % 8 == 0 && cols % 8 == 0 && ld * 2 <= kMaxPitch;
}

struct LossSpace {
  char *x, *w;
  int *ex, *ew;
  float2 *parts;
  float *picked;
  int64_t count;
  LossSpace(Carver &c, const Sizes &s) {
    x = c.take<char>(s.packed(s.rows));
    w = c.take<char>(s.packed(s.classes));
    ex = c.take<int>(s.rows);
    ew = c.take<int>(s.classes);
    count = ceil_div(s.classes, kWaveCols[s.loss().shape]);
    parts = c.take<float2>(s.rows * count);
    picked = c.take<float>(s.rows);
  }
};

struct GradSpace {
  char *x, *w, *xg, *g;
  Scalars *scalars;
  float *dx, *dw;
  GradSpace(Carver &c, const Sizes &s) {
    scalars = c.take<Scalars>(1);
    x = c.take<char>(s.packed(s.rows));
    w = c.take<char>(s.packed(s.classes));
    xg = c.take<char>(s.dtype == SDNN_FP32 ? s.packed(s.rows) : 0);
    g = c.take<char>((size_t)(s.rows * s.g_pitch()));
    dx = c.take<float>(s.dx().splits > 1 || s.piece() < s.classes ? (size_t)(s.dx().splits * s.rows * s.ld_slab()) : 0);
    size_t most = 0;
    for (int64_t n : {s.piece(), s.classes % std::max<int64_t>(1, s.piece())}) {
      const Plan p = s.dw(n);
      if (n > 0 && p.splits > 1) most = std::max(most, (size_t)(p.splits * n * s.ld_slab()));
    }
    dw = c.take<float>(most);
  }
};

unsigned row_grid(int64_t rows) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(rows, 2048)); }

// A matrix as an operand: in place, or copied into `space` first.
template <int KIND>
Matrix operand(const void *data, int64_t ld, int64_t rows, const Sizes &s, const int64_t *labels, const float *top, int *exponents, const float *weights, char *space, hipStream_t stream) {
  if constexpr (KIND == KIND_BF16) {
    if (!labels && usable_in_place(data, ld, s.features)) return {(const char *)data, ld * 2, rows, s.features * 2, 0};
    const bool vec = ((uintptr_t)data & 15) == 0 && ld % 8 == 0;
    if (rows)
      hipLaunchKernelGGL(k_copy_rows, dim3(row_grid(rows)), dim3(256), 0, stream, (const __bf16 *)data, ld, rows, s.features, s.pitch_values(), labels, s.classes, vec, (__bf16 *)space);
    return {space, s.pitch_values() * 2, rows, s.pitch_values() * 2, 0};
  } else {
    if (rows)
      hipLaunchKernelGGL(k_split_rows, dim3(row_grid(rows)), dim3(256), 0, stream, (const float *)data, ld, rows, s.features, s.groups(), labels, s.classes, weights, top, exponents, space);
    return {space, s.groups() * 128, rows, s.groups() * 128, 0};
  }
}

template <int KIND>
sdnn_status loss_of(const Sizes &s, const void *x, int64_t ldx, const void *w, int64_t ldw, const int64_t *labels, float *loss, float *lse, void *workspace, hipStream_t stream) {
  Carver carver{(char *)workspace};
  const LossSpace sp(carver, s);
  const Matrix a = operand<KIND>(x, ldx, s.rows, s, nullptr, nullptr, sp.ex, nullptr, sp.x, stream);
  const Matrix b = operand<KIND>(w, ldw, s.classes, s, nullptr, nullptr, sp.ew, nullptr, sp.w, stream);
  sdnn_status st = launched("rows");
  if (st != SDNN_OK) return st;
  const LossParts<KIND> e{{sp.ex, sp.ew, nullptr, nullptr}, labels, s.rows, s.classes, sp.parts, sp.count, sp.picked};
  st = run_shape<KIND, false, false>(s.loss(), a, b, s.rows, s.classes, s.features, e, stream, "loss");
  if (st != SDNN_OK) return st;
  hipLaunchKernelGGL(k_loss, dim3((unsigned)ceil_div(s.rows, 4)), dim3(256), 0, stream, sp.parts, sp.count, sp.picked, labels, s.rows, s.classes, loss, lse);
  return launched("loss");
}

// C = A B^T over k, into `to` directly or through fp32 slabs.
template <int KIND, bool AA, class T>
sdnn_status product(const Plan &p, const Matrix &a, const Matrix &b, int64_t k, float *slabs, int64_t ld_slab, bool through, bool add, bool last, const Store<T> &to, hipStream_t stream, const char *what) {
  if (!through) return run_shape<KIND, AA, true>(p, a, b, to.rows, to.cols, k, to, stream, what);
  const Accumulate e{slabs, ld_slab, to.rows, to.cols, add};
  sdnn_status st = run_shape<KIND, AA, true>(p, a, b, to.rows, to.cols, k, e, stream, what);
  if (st != SDNN_OK || !last) return st;
  const int64_t work = ceil_div(to.rows * (ld_slab / 4), 256);
  hipLaunchKernelGGL((k_sum_slabs<T>), dim3((unsigned)std::min<int64_t>(work, 8192)), dim3(256), 0, stream, slabs, p.splits, ld_slab, to);
  return launched(what);
}

template <class T>
bool vector_rows(const T *p, int64_t ld) {
  return (uintptr_t)p % (4 * sizeof(T)) == 0 && ld % 4 == 0;
}

template <class T>
__global__ __launch_bounds__(256) void k_zero_rows(T *out, int64_t ld, int64_t rows, int64_t cols) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < cols; c += 256) out[r * ld + c] = (T)0.0f;
}

template <int KIND, class T>
sdnn_status grad_of(const Sizes &s, const T *x, int64_t ldx, const T *w, int64_t ldw, const int64_t *labels, const float *lse, const float *weights, T *dx, int64_t lddx, T *dw, int64_t lddw,
                    void *workspace, hipStream_t stream) {
  Carver carver{(char *)workspace};
  const GradSpace sp(carver, s);
  if (s.rows == 0) {
    if (dw) hipLaunchKernelGGL((k_zero_rows<T>), dim3(row_grid(s.classes)), dim3(256), 0, stream, dw, lddw, s.classes, s.features);
    return launched("gradient");
  }
  hipLaunchKernelGGL(k_count, dim3(1), dim3(1024), 0, stream, labels, s.rows, s.classes, sp.scalars);
  float *top_x = nullptr, *top_w = nullptr;
  if constexpr (KIND == KIND_SPLIT) {
    top_x = sp.scalars->top[0];
    top_w = sp.scalars->top[1];
    hipLaunchKernelGGL(k_top, dim3(kTopBlocks), dim3(256), 0, stream, x, ldx, s.rows, s.features, labels, s.classes, (const float *)nullptr, top_x);
    hipLaunchKernelGGL(k_top, dim3(kTopBlocks), dim3(256), 0, stream, w, ldw, s.classes, s.features, (const int64_t *)nullptr, s.classes, (const float *)nullptr, top_w);
  }
  const Matrix a = operand<KIND>(x, ldx, s.rows, s, labels, top_x, nullptr, nullptr, sp.x, stream);
  const Matrix b = operand<KIND>(w, ldw, s.classes, s, nullptr, top_w, nullptr, nullptr, sp.w, stream);
  Matrix ag = a;  // dw's other operand: the rows, in fp32 times their weights (in bf16 G holds the weights)
  const float *top_g = top_x;
  if (KIND == KIND_SPLIT && weights && dw) {
    float *top = sp.scalars->top[2];
    hipLaunchKernelGGL(k_top, dim3(kTopBlocks), dim3(256), 0, stream, (const float *)x, ldx, s.rows, s.features, labels, s.classes, weights, top);
    ag = operand<KIND>(x, ldx, s.rows, s, labels, top, nullptr, weights, sp.xg, stream);
    top_g = top;
  }
  sdnn_status st = launched("gradient");
  const float *mean = KIND == KIND_SPLIT && !weights ? &sp.scalars->mean : nullptr;
  const float *row_weights = KIND == KIND_SPLIT ? weights : nullptr;
  const Plan px = s.dx();
  const int64_t piece = s.piece();
  const bool through_x = px.splits > 1 || piece < s.classes;
  for (int64_t v0 = 0; v0 < s.classes && st == SDNN_OK; v0 += piece) {
    const int64_t n = std::min(piece, s.classes - v0);
    const bool last = v0 + n == s.classes;
    Matrix wp = b;
    wp.data += v0 * b.pitch;
    wp.rows = n;
    const WriteGrad<KIND> e{{nullptr, nullptr, top_x, top_w}, labels, lse, weights, sp.scalars, s.rows, s.classes, v0, n, sp.g, s.g_pitch()};
    st = run_shape<KIND, false, false>(s.logits(n), a, wp, s.rows, n, s.features, e, stream, "gradient");
    if (st != SDNN_OK) return st;
    const int64_t wide = KIND == KIND_SPLIT ? ceil_div(n, 32) * 128 : ceil_div(n, 8) * 16;  // bytes of a row of G
    if (dx) {
      const Store<T> to{dx, lddx, s.rows, s.features, vector_rows(dx, lddx), {row_weights, mean, top_w}};
      st = product<KIND, false>(px, Matrix{sp.g, s.g_pitch(), s.rows, wide, 0}, wp, n, sp.dx, s.ld_slab(), through_x, v0 > 0, last, to, stream, "gradient of the rows");
      if (st != SDNN_OK) return st;
    }
    if (dw) {
      const Plan pw = s.dw(n);
      const Store<T> to{dw + v0 * lddw, lddw, n, s.features, vector_rows(dw + v0 * lddw, lddw), {nullptr, mean, top_g}};
      st = product<KIND, true>(pw, Matrix{sp.g, s.g_pitch(), s.rows, wide, 0}, ag, s.rows, sp.dw, s.ld_slab(), pw.splits > 1, false, true, to, stream, "gradient of the weights");
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
  if ((st = check_workspace(workspace, workspace_bytes, sdnn_readout_workspace_bytes(n_rows, n_classes, n_features, dtype, 0))) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  return dtype == SDNN_BF16 ? loss_of<KIND_BF16>(s, x, ldx, w, ldw, labels, loss, lse, workspace, stream) : loss_of<KIND_SPLIT>(s, x, ldx, w, ldw, labels, loss, lse, workspace, stream);
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
  if ((st = check_workspace(workspace, workspace_bytes, sdnn_readout_workspace_bytes(n_rows, n_classes, n_features, dtype, 1))) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (dtype == SDNN_BF16)
    return grad_of<KIND_BF16, __bf16>(s, (const __bf16 *)x, ldx, (const __bf16 *)w, ldw, labels, lse, row_grad, (__bf16 *)dx, lddx, (__bf16 *)dw, lddw, workspace, stream);
  return grad_of<KIND_SPLIT, float>(s, (const float *)x, ldx, (const float *)w, ldw, labels, lse, row_grad, (float *)dx, lddx, (float *)dw, lddw, workspace, stream);
}

}  // extern "C"
