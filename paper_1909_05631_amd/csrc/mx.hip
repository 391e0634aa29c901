// Microscaled 4-bit floating point: quantisation, its inverse, and the product of quantised rows.
//
// A row of n values is held in blocks of 32: one byte of scale s (the power of two 2^(s - 127)) and 16 bytes of codes,
// two to a byte, the even value in the low half. A code is a sign bit and a magnitude of {0, .5, 1, 1.5, 2, 3, 4, 6}.
// A block's scale is 2^(floor(log2 max|x|) - 2), which puts its largest value in [4, 8); values are rounded to the
// nearest code, ties to the even one, and at most 6. A block with an infinity or a NaN has scale 255 and stands for NaN.
// Rows are padded to whole runs of 4 blocks (128 values, one matrix instruction) with zero codes.
//
// The product runs on the scaled 4-bit matrix instructions (16 x 16 x 128, fp32 sums of exact products): 64 bytes
// of a row are 4 lane groups' 16-byte blocks, and each lane hands the instruction its block's scale byte.
#include "dense.h"

using namespace dense;
using tile::KIND_MX;

namespace {

constexpr int kNanScale = 255;

__host__ __device__ inline int64_t blocks_of(int64_t n) { return 4 * ceil_div(n, 128); }

// Magnitude code of a >= 0: the grid's middles, ties to the even code.
__device__ __forceinline__ uint32_t code_of(float a) {
  return (uint32_t)(a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
}

// Eight values' codes and, from the four lanes of a block together, the block's scale byte.
__device__ __forceinline__ uint32_t quantize8(const float (&v)[8], uint32_t &scale) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t b = __float_as_uint(v[i]) & 0x7fffffffu;
    top = b > top ? b : top;
  }
#pragma unroll
  for (int d = 1; d < 4; d <<= 1) {
    const uint32_t o = __shfl_xor(top, d);
    top = o > top ? o : top;
  }
  if (top >= 0x7f800000u) {
    scale = kNanScale;
    return 0;
  }
  const uint32_t field = top >> 23;
  scale = field > 2 ? field - 2 : 0;
  const float inverse = __uint_as_float((254 - scale) << 23);  // 2^(127 - scale), exact
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) codes |= (code_of(fabsf(v[i] * inverse)) | (__float_as_uint(v[i]) >> 31) << 3) << (4 * i);
  return codes;
}

template <class T>
__device__ __forceinline__ void load8(const T *row, int64_t k, int64_t n, bool vec, float (&v)[8]) {
  typedef T T8 __attribute__((ext_vector_type(8)));
  if (vec && k + 8 <= n) {
    const T8 x = *(const T8 *)(row + k);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = k + i < n ? (float)row[k + i] : 0.0f;
  }
}

// Eight values a lane, four lanes a block. Bound by memory: 4 (or 2) bytes read and 17/32 written a value.
template <class T>
__global__ __launch_bounds__(256) void k_quantize(const T *x, int64_t ld, int64_t rows, int64_t n, int64_t blocks, bool vec, uint8_t *codes, uint8_t *scales) {
  const int per = (int)blocks * 4;  // a multiple of 16: a block's lanes stay together
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const T *row = x + r * ld;
    uint8_t *to = codes + r * blocks * 16, *scale_to = scales + r * blocks;
    for (int c = blockIdx.x * 256 + threadIdx.x; c < per; c += gridDim.x * 256) {
      float v[8];
      load8(row, c * 8, n, vec, v);
      uint32_t scale;
      *(uint32_t *)(to + c * 4) = quantize8(v, scale);
      if ((c & 3) == 0) scale_to[c >> 2] = (uint8_t)scale;
    }
  }
}

__device__ __forceinline__ float value_of(uint32_t code, uint32_t scale) {
  // the magnitude as a float: codes 2 ... 7 are 1.m 2^(e-1) with two bits of e and one of m, code 1 is a half
  const uint32_t m = code & 7;
  const float a = m < 2 ? 0.5f * m : __uint_as_float((126 + (m >> 1)) << 23 | (m & 1) << 22);
  const float v = ldexpf(code & 8 ? -a : a, (int)scale - 127);
  return scale == kNanScale ? __builtin_nanf("") : v;
}

template <class T>
__global__ __launch_bounds__(256) void k_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t n, int64_t blocks, T *out, int64_t ld, bool vec) {
  const int per = (int)ceil_div(n, 8);
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const uint8_t *from = codes + r * blocks * 16, *scale_of = scales + r * blocks;
    for (int c = blockIdx.x * 256 + threadIdx.x; c < per; c += gridDim.x * 256) {
      const uint32_t word = *(const uint32_t *)(from + c * 4), scale = scale_of[c >> 2];
      f32x4 v[2];
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j >> 2][j & 3] = value_of(word >> (4 * j) & 15, scale);
      T *to = out + r * ld + c * 8;
      const int left = min((int)n - c * 8, 8);
      store4(to, v[0], left < 4 ? left : 4, vec);
      if (left > 4) store4(to + 4, v[1], left - 4, vec);
    }
  }
}

template <class T>
struct Store {
  T *out;
  int64_t ld, rows, cols;
  bool vec;
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t r = row0 + 16 * i + (threadIdx.x & 15);
      store_row<T, B::kTN>(out + r * ld, col0, cols, vec, r < rows, [&](int j) { return block.acc[i][j]; });
    }
  }
};

template <class T>
sdnn_status product(const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes, const uint8_t *w_scales, int64_t rows, int64_t outputs, int64_t n, T *out, int64_t ld, hipStream_t stream) {
  const int64_t pitch = blocks_of(n) * 16;
  const Matrix a{(const char *)x_codes, pitch, rows, pitch, 0, x_scales}, b{(const char *)w_codes, pitch, outputs, pitch, 0, w_scales};
  const Store<T> e{out, ld, rows, outputs, (uintptr_t)out % 16 == 0 && ld * sizeof(T) % 16 == 0};
  return run_shape<KIND_MX, false, false>(plan(KIND_MX, rows, outputs, n, 1, kAlong), a, b, rows, outputs, n, e, stream, "product");
}

// Workgroups along a row of `items` lanes, and down the rows: 16 to 32 a CU where there is work for them.
dim3 grid_of(int64_t rows, int64_t items) {
  const int64_t x = ceil_div(items, 256);
  return dim3((unsigned)x, (unsigned)std::max<int64_t>(1, std::min<int64_t>({rows, 65535, ceil_div(kCus * 32, x)})));
}

template <class T>
sdnn_status quantize(const T *x, int64_t ld, int64_t rows, int64_t n, uint8_t *codes, uint8_t *scales, hipStream_t stream) {
  const int64_t blocks = blocks_of(n);
  const bool vec = (uintptr_t)x % 16 == 0 && ld * sizeof(T) % 16 == 0;
  hipLaunchKernelGGL((k_quantize<T>), grid_of(rows, blocks * 4), dim3(256), 0, stream, x, ld, rows, n, blocks, vec, codes, scales);
  return launched("quantize");
}

sdnn_status check_mx(const char *name, const uint8_t *codes, const uint8_t *scales) {
  if (!codes || !scales) return fail(SDNN_EINVAL, "the codes or scales of %s are null", name);
  if (((uintptr_t)codes & 15) || ((uintptr_t)scales & 3)) return fail(SDNN_EINVAL, "the codes of %s are not 16-byte aligned, or its scales not 4-byte aligned", name);
  return SDNN_OK;
}

sdnn_status check_shape(int64_t n_rows, int64_t n_values, int32_t dtype) {
  if (n_rows < 0 || n_rows > kMaxRows) return fail(SDNN_EINVAL, "n_rows %lld is outside [0, %lld]", (long long)n_rows, (long long)kMaxRows);
  if (n_values < 1 || n_values > kMaxFeatures) return fail(SDNN_EINVAL, "n_values %lld is outside [1, %lld]", (long long)n_values, (long long)kMaxFeatures);
  if (!good_dtype(dtype)) return fail(SDNN_EINVAL, "dtype %d is neither SDNN_FP32 nor SDNN_BF16", dtype);
  return SDNN_OK;
}

sdnn_status check_outputs(int64_t n_outputs) {
  if (n_outputs < 0 || n_outputs > kMaxClasses) return fail(SDNN_EINVAL, "n_outputs %lld is outside [0, %lld]", (long long)n_outputs, (long long)kMaxClasses);
  return SDNN_OK;
}

}  // namespace

extern "C" {

int64_t sdnn_mx_blocks(int64_t n_values) { return n_values < 1 || n_values > kMaxFeatures ? 0 : blocks_of(n_values); }

sdnn_status sdnn_mx_quantize(const void *x, int64_t ldx, int32_t dtype, int64_t n_rows, int64_t n_values, uint8_t *codes, uint8_t *scales, void *hip_stream) {
  sdnn_status st = check_shape(n_rows, n_values, dtype);
  if (st != SDNN_OK || n_rows == 0) return st;
  if ((st = check_matrix("x", x, ldx, n_values, dtype)) != SDNN_OK) return st;
  if ((st = check_mx("x", codes, scales)) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  return dtype == SDNN_BF16 ? quantize((const __bf16 *)x, ldx, n_rows, n_values, codes, scales, stream) : quantize((const float *)x, ldx, n_rows, n_values, codes, scales, stream);
}

sdnn_status sdnn_mx_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t n_rows, int64_t n_values, void *out, int64_t ldo, int32_t dtype, void *hip_stream) {
  sdnn_status st = check_shape(n_rows, n_values, dtype);
  if (st != SDNN_OK || n_rows == 0) return st;
  if ((st = check_matrix("out", out, ldo, n_values, dtype)) != SDNN_OK) return st;
  if ((st = check_mx("the input", codes, scales)) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const int64_t blocks = blocks_of(n_values);
  const dim3 grid = grid_of(n_rows, ceil_div(n_values, 8));
  const bool vec = (uintptr_t)out % (4 * dtype_bytes(dtype)) == 0 && ldo % 4 == 0;
  if (dtype == SDNN_BF16)
    hipLaunchKernelGGL((k_dequantize<__bf16>), grid, dim3(256), 0, stream, codes, scales, n_rows, n_values, blocks, (__bf16 *)out, ldo, vec);
  else
    hipLaunchKernelGGL((k_dequantize<float>), grid, dim3(256), 0, stream, codes, scales, n_rows, n_values, blocks, (float *)out, ldo, vec);
  return launched("dequantize");
}

sdnn_status sdnn_mx_product(const uint8_t *x_codes, const uint8_t *x_scales, const uint8_t *w_codes, const uint8_t *w_scales, int64_t n_rows, int64_t n_outputs, int64_t n_values, void *out,
                            int64_t ldo, int32_t dtype, void *hip_stream) {
  sdnn_status st = check_shape(n_rows, n_values, dtype);
  if (st == SDNN_OK) st = check_outputs(n_outputs);
  if (st != SDNN_OK || n_rows == 0 || n_outputs == 0) return st;
  if ((st = check_mx("x", x_codes, x_scales)) != SDNN_OK) return st;
  if ((st = check_mx("w", w_codes, w_scales)) != SDNN_OK) return st;
  if ((st = check_matrix("out", out, ldo, n_outputs, dtype)) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  return dtype == SDNN_BF16 ? product(x_codes, x_scales, w_codes, w_scales, n_rows, n_outputs, n_values, (__bf16 *)out, ldo, stream)
                            : product(x_codes, x_scales, w_codes, w_scales, n_rows, n_outputs, n_values, (float *)out, ldo, stream);
}

size_t sdnn_mx_linear_workspace_bytes(int64_t n_rows, int64_t n_values) {
  if (n_rows < 0 || n_rows > kMaxRows || n_values < 1 || n_values > kMaxFeatures) return 0;
  Carver c{nullptr};
  c.take<uint8_t>((size_t)(n_rows * blocks_of(n_values) * 16));
  c.take<uint8_t>((size_t)(n_rows * blocks_of(n_values)));
  return c.used;
}

sdnn_status sdnn_mx_linear(const void *x, int64_t ldx, int32_t dtype, const uint8_t *w_codes, const uint8_t *w_scales, int64_t n_rows, int64_t n_outputs, int64_t n_values, void *out, int64_t ldo,
                           void *workspace, size_t workspace_bytes, void *hip_stream) {
  sdnn_status st = check_shape(n_rows, n_values, dtype);
  if (st == SDNN_OK) st = check_outputs(n_outputs);
  if (st != SDNN_OK || n_rows == 0 || n_outputs == 0) return st;
  if ((st = check_matrix("x", x, ldx, n_values, dtype)) != SDNN_OK) return st;
  if ((st = check_mx("w", w_codes, w_scales)) != SDNN_OK) return st;
  if ((st = check_matrix("out", out, ldo, n_outputs, dtype)) != SDNN_OK) return st;
  if ((st = check_workspace(workspace, workspace_bytes, sdnn_mx_linear_workspace_bytes(n_rows, n_values))) != SDNN_OK) return st;
  Carver c{(char *)workspace};
  uint8_t *codes = c.take<uint8_t>((size_t)(n_rows * blocks_of(n_values) * 16)), *scales = c.take<uint8_t>((size_t)(n_rows * blocks_of(n_values)));
  if ((st = sdnn_mx_quantize(x, ldx, dtype, n_rows, n_values, codes, scales, hip_stream)) != SDNN_OK) return st;
  return sdnn_mx_product(codes, scales, w_codes, w_scales, n_rows, n_outputs, n_values, out, ldo, dtype, hip_stream);
}

}  // extern "C"
