// Orthogonalising an update by Newton-Schulz products (batches of rows x cols matrices):
//
//   X = G / (||G||_F + eps);  `steps` times: A = X X^T, X <- a X + (b A + c A A) X      (rows <= cols)
//                                            A = X^T X, X <- X (a + b A + c A A)        (rows > cols: the same X)
//
// so that A is square in the smaller size and X is never transposed. Every product runs on the fp16 matrix cores with
// each factor held as two fp16 parts (KIND_SPLIT of tile.h), which keeps fp32's exactness at 3 fp16 products each.
// A and A A are symmetric: only blocks on and above the diagonal are computed, and written to both places.
// Each step is three launches; their epilogues apply a, b, c and write the next factor in its two parts.
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
  double *parts;
  Info *info;
  char *x[2], *a, *b;
  Space(Carver &c, int64_t batch, int64_t rows, int64_t cols) {
    const int64_t m = std::min(rows, cols);
    parts = c.take<double>((size_t)(batch * kNormBlocks));
    info = c.take<Info>((size_t)batch);
    for (char *&p : x) p = c.take<char>((size_t)(batch * rows * ceil_div(cols, 32) * 128));
    a = c.take<char>((size_t)(batch * m * ceil_div(m, 32) * 128));
    b = c.take<char>((size_t)(batch * m * ceil_div(m, 32) * 128));
  }
};

template <class T>
sdnn_status orthogonalize(const T *g, int64_t ldg, int64_t batch_g, T *out, int64_t ldo, int64_t batch_o, int64_t batch, int64_t rows, int64_t cols, int steps, const float *coef, float eps,
                          void *workspace, hipStream_t stream) {
  Carver carver{(char *)workspace};
  const Space sp(carver, batch, rows, cols);
  const Source<T> src{g, ldg, batch_g, rows, cols};
  const unsigned norm_blocks = (unsigned)std::min<int64_t>(rows, kNormBlocks), row_blocks = (unsigned)std::min<int64_t>(rows, 2048);
  hipLaunchKernelGGL((k_squares<T>), dim3(norm_blocks, (unsigned)batch), dim3(256), 0, stream, src, sp.parts);
  if (steps == 0) {
    hipLaunchKernelGGL((k_scale<T>), dim3(row_blocks, (unsigned)batch), dim3(256), 0, stream, src, sp.parts, (int)norm_blocks, (double)eps, out, ldo, batch_o);
    return launched("orthogonalize");
  }
  Bound bounds[kMaxSteps + 1];
  double u = 1.0, l = 1.0;
  for (int k = 0; k <= steps; ++k) {
    bounds[k] = {(float)std::log2(u), (float)std::log2(l)};
    double value, slope;
    reach(coef[0], coef[1], coef[2], u, value, slope);
    u = std::min(1e30, std::max(1e-30, 1.01 * value));  // what rounding adds is far below a hundredth
    l = std::min(1e30, std::max(1e-30, 1.01 * slope * l));
  }
  const int64_t pitch = ceil_div(cols, 32) * 128, m = std::min(rows, cols), square = ceil_div(m, 32) * 128;
  hipLaunchKernelGGL((k_start<T>), dim3(row_blocks, (unsigned)batch), dim3(256), 0, stream, src, sp.parts, (int)norm_blocks, (double)eps, bounds[0], sp.info, sp.x[0], pitch);
  sdnn_status st = launched("orthogonalize");
  const bool tall = rows > cols;
  const Plan gram = plan(KIND_SPLIT, m, m, std::max(rows, cols), 1, tall ? kAnyForm : kAlong, batch, true);
  const Plan power = plan(KIND_SPLIT, m, m, m, 1, kAlong, batch, true);
  const Plan update = plan(KIND_SPLIT, rows, cols, m, 1, tall ? kAlong : kAnyForm, batch);
  for (int k = 0; k < steps && st == SDNN_OK; ++k) {
    const char *x = sp.x[k & 1];
    char *next = k + 1 < steps ? sp.x[(k + 1) & 1] : nullptr;
    const Matrix mx{x, pitch, rows, pitch, rows * pitch}, ma{sp.a, square, m, square, m * square}, mb{sp.b, square, m, square, m * square};
    Square e{nullptr, sp.a, m, square, coef[1], coef[2], bounds[k], sp.info};
    st = tall ? run_shape<KIND_SPLIT, true, true>(gram, mx, mx, m, m, rows, e, stream, "orthogonalize", true, (int)batch)
              : run_shape<KIND_SPLIT, false, false>(gram, mx, mx, m, m, cols, e, stream, "orthogonalize", true, (int)batch);
    if (st != SDNN_OK) return st;
    e.a = sp.a;
    e.out = sp.b;
    st = run_shape<KIND_SPLIT, false, false>(power, ma, ma, m, m, m, e, stream, "orthogonalize", true, (int)batch);
    if (st != SDNN_OK) return st;
    const Update<T> last{x, next, out, ldo, batch_o, rows, cols, pitch, (uintptr_t)out % (4 * sizeof(T)) == 0 && ldo % 4 == 0 && batch_o % 4 == 0, coef[0], coef[1], coef[2], bounds[k], bounds[k + 1], sp.info};
    st = tall ? run_shape<KIND_SPLIT, false, false>(update, mx, mb, rows, cols, m, last, stream, "orthogonalize", false, (int)batch)
              : run_shape<KIND_SPLIT, false, true>(update, mb, mx, rows, cols, m, last, stream, "orthogonalize", false, (int)batch);
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
