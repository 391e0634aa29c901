// Microscaled 4-bit floating point: quantisation, its inverse, and the product of quantised rows.
//
// A row of n values is held in blocks of 32: one byte of scale s (the power of two 2^(s - 127)) and 16 bytes of codes,
// two to a byte, the even value in the low half. A code is a sign bit and a magnitude of {0, .5, 1, 1.5, 2, 3, 4, 6}.
// A block's scale is 2^(floor(log2 max|x|) - 2), which puts its largest value in [4, 8); values are rounded to the
// nearest code, ties to the even one, and at most 6. A block with an infinity or a NaN has scale 255 and stands for NaN.
// Rows are padded to whole runs of 4 blocks (128 values, one matrix instruction) with zero codes.
//
// The product runs on the scaled 4-bit matrix instructions (16 x 16 x 128, fp32 sums of exact products): 64 bytes
// of a row are 4 lane groups' 16-byte blocks, and each lane hands the instruction its block's scale byte. 4096 x 16384
// x 16384: 535 us with its quantisation once the card's clock has settled, 4.1 PFLOP/s (up to 680 in the first passes).
#include "dense.h"

using namespace dense;
using tile::KIND_MX;

namespace {

constexpr int kNanScale = 255;

__host__ __device__ inline int64_t blocks_of(int64_t n) { return 4 * ceil_div(n, 128); }

// Eight values' codes and, from the four lanes of a block together, the block's scale byte. The values are multiplied by
// a power of two, exactly; the conversion instruction rounds to nearest, ties to even, and saturates.
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
  const bool bad = top >= 0x7f800000u;
  const uint32_t field = top >> 23;
  scale = bad ? kNanScale : field > 2 ? field - 2 : 0;
  const float inverse = bad ? 0.0f : __uint_as_float((254 - scale) << 23);  // 2^(127 - scale)
  uint32_t codes = 0;
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[0] * inverse, v[1] * inverse, 1.0f, 0);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[2] * inverse, v[3] * inverse, 1.0f, 1);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[4] * inverse, v[5] * inverse, 1.0f, 2);
  codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, v[6] * inverse, v[7] * inverse, 1.0f, 3);
  return bad ? 0 : codes;
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

// Eight values a lane, four lanes a block. Bound by memory, 4 (or 2) bytes read and 17/32 written a value: 8192 x 16384
// fp32 118 us (5.1 TB/s) over and over, 149 after other work; bf16 62 us.
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

// Byte BYTE's two values.
template <int BYTE>
__device__ __forceinline__ void values_of(uint32_t word, float scale, float *v) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  const f32x2 two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, 1.0f, BYTE);
  v[0] = two[0] * scale;
  v[1] = two[1] * scale;
}
__device__ __forceinline__ float scale_of(uint32_t s) {
  return s == kNanScale ? __builtin_nanf("") : __uint_as_float(s ? s << 23 : 1u << 22);  // 2^-127 is not normal
}

// 16 bytes of values a lane: a wave stores a run of 1024. Bound by memory, most of it the values written: 8192 x 16384 fp32
// 124 to 141 us (4.9 to 4.3 TB/s), bf16 68 us.
template <class T>
__global__ __launch_bounds__(256) void k_dequantize(const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t n, int64_t blocks, T *out, int64_t ld, bool vec) {
  constexpr int kEach = 16 / sizeof(T);
  const int per = (int)ceil_div(n, kEach);
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const uint8_t *from = codes + r * blocks * 16, *scales_from = scales + r * blocks;
    for (int c = blockIdx.x * 256 + threadIdx.x; c < per; c += gridDim.x * 256) {
      const float scale = scale_of(scales_from[c * kEach / 32]);
      float v[kEach];
      uint32_t word;
      if constexpr (kEach == 8)
        word = *(const uint32_t *)(from + c * 4);
      else
        word = *(const uint16_t *)(from + c * 2);
      values_of<0>(word, scale, v);
      values_of<1>(word, scale, v + 2);
      if constexpr (kEach == 8) {
        values_of<2>(word, scale, v + 4);
        values_of<3>(word, scale, v + 6);
      }
      typedef T Out __attribute__((ext_vector_type(kEach)));
      Out o;
#pragma unroll
      for (int k = 0; k < kEach; ++k) o[k] = (T)v[k];
      T *to = out + r * ld + (int64_t)c * kEach;
      const int left = min((int)n - c * kEach, kEach);
      if (vec && left == kEach) {
        *(Out *)to = o;
      } else {
#pragma unroll
        for (int k = 0; k < kEach; ++k)
          if (k < left) to[k] = o[k];
      }
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

// Few rows: one launch that quantises x into LDS, every workgroup for itself, and streams w from memory to the matrix
// instructions, each byte once and without LDS. A workgroup takes 16 outputs at a time and its four waves share k, 1024
// values of a wave on their way at once; their sums meet in LDS. Bound by w's bytes: 65536 x 4096 (143 MB) takes 28.6 us
// for one row, 5.0 TB/s. Every workgroup's own quantisation is what limits it, by the row: 16 rows of 4096 cost 10 us
// more than one. Measured against the tiles with their quantisation (us here / there, w not in the caches):
//   up to 4 rows, whatever their length: 1 x 65536 to 4096 outputs 46/107, 4 x 16384 27/32; 1 x 8192 to 65536 outputs 54/65,
//     4 x 8192 63/66, 4 x 16384 120/115 (the worst: 4 x 1024 to 65536 outputs 15/13);
//   more rows, few values: 16 x 256 to 65536 outputs 9/12 (but 6 x 1024 15/13);
//   more rows, few outputs, where the tiles would be a few long chains of k: 8 x 4096 to 4096 outputs 11.7/12.6, 16 x 2048
//     11.4/11.8, but 12 x 4096 15/12, and 8 x 4096 to 20000 outputs 21/18.
constexpr int kFewRows = 16, kFewValues = 65536;
inline bool is_few(int64_t rows, int64_t outputs, int64_t n) {
  const int64_t values = rows * ceil_div(n, 256) * 256;
  if (rows > kFewRows || values > kFewValues) return false;
  return rows <= 4 || values <= 4096 || (values <= 32768 && outputs <= 32 * kCus);
}

template <class T>
__global__ __launch_bounds__(256) void k_few(const T *x, int64_t ldx, bool vec_x, int rows, int n, const uint8_t *w_codes, const uint8_t *w_scales, int64_t outputs, T *out, int64_t ldo, bool vec) {
  using tile::i32x4;
  __shared__ __attribute__((aligned(16))) uint8_t codes[kFewValues / 2];
  __shared__ __attribute__((aligned(16))) uint8_t scales[kFewValues / 32];
  __shared__ f32x4 sums[4][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tile::uniform(tid >> 6), i16 = lane & 15, j4 = lane >> 4;
  const int blocks = (int)blocks_of(n), slabs = (blocks + 7) / 8, wide = slabs * 8;  // blocks of a row: in memory, in LDS
  const int64_t pitch = (int64_t)blocks * 16;
  for (int i = tid; i < rows * wide * 4; i += 256) {
    const int r = i / (wide * 4), c = i - r * (wide * 4);
    float v[8];
    load8(x + r * ldx, (int64_t)c * 8, n, vec_x, v);
    uint32_t scale;
    *(uint32_t *)(codes + i * 4) = quantize8(v, scale);
    if ((c & 3) == 0) scales[i >> 2] = (uint8_t)scale;
  }
  __syncthreads();
  const int per = (slabs + 3) / 4, s0 = wave * per, s1 = min(s0 + per, slabs);  // this wave's k
  const bool mine = i16 < rows;
  for (int64_t first = (int64_t)blockIdx.x * 16; first < outputs; first += (int64_t)gridDim.x * 16) {
    const int there = outputs - first < 16 ? (int)(outputs - first) : 16;
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void *)(w_codes + first * pitch), 0, there * (int)pitch, 0x00027000);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)(w_scales + first * blocks), 0, there * blocks, 0x00027000);
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s = s0; s < s1; s += 4) {
      i32x4 b[4][2];
      int sb[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int block = (s + u) * 8 + 2 * j4;
        const bool in = s + u < s1 && block < blocks;  // past them: zeros
#pragma unroll
        for (int q = 0; q < 2; ++q) b[u][q] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, in ? i16 * (int)pitch + (block + q) * 16 : tile::kOut, 0, 0));
        sb[u] = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, in ? i16 * blocks + block : tile::kOut, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int at = (i16 * wide + min(s + u, slabs - 1) * 8 + 2 * j4);
        i32x4 a[2] = {};
        int sa = 0;
        if (mine) {
          a[0] = *(const i32x4 *)(codes + at * 16);
          a[1] = *(const i32x4 *)(codes + at * 16 + 16);
          sa = *(const uint16_t *)(scales + at);
        }
        acc = tile::mfma_mx<0>(b[u][0], a[0], acc, sb[u], s + u < s1 ? sa : 0);
        acc = tile::mfma_mx<1>(b[u][1], a[1], acc, sb[u], s + u < s1 ? sa : 0);
      }
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
      const f32x4 v = sums[0][lane] + sums[1][lane] + sums[2][lane] + sums[3][lane];
      const int64_t c = first + 4 * j4;
      if (mine && c < outputs) store4(out + i16 * ldo + c, v, (int)(outputs - c < 4 ? outputs - c : 4), vec);
    }
    __syncthreads();
  }
}

template <class T>
sdnn_status few(const T *x, int64_t ldx, const uint8_t *w_codes, const uint8_t *w_scales, int64_t rows, int64_t outputs, int64_t n, T *out, int64_t ldo, hipStream_t stream) {
  const bool vec_x = (uintptr_t)x % 16 == 0 && ldx * sizeof(T) % 16 == 0, vec = (uintptr_t)out % (4 * sizeof(T)) == 0 && ldo % 4 == 0;
  hipLaunchKernelGGL((k_few<T>), dim3((unsigned)std::min<int64_t>(ceil_div(outputs, 16), 4 * kCus)), dim3(256), 0, stream, x, ldx, vec_x, (int)rows, (int)n, w_codes, w_scales, outputs, out, ldo, vec);
  return launched("linear");
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
  const dim3 grid = grid_of(n_rows, ceil_div(n_values, 16 / dtype_bytes(dtype)));
  const bool vec = (uintptr_t)out % 16 == 0 && ldo * dtype_bytes(dtype) % 16 == 0;
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
  if (is_few(n_rows, n_outputs, n_values)) {
    const hipStream_t stream = (hipStream_t)hip_stream;
    return dtype == SDNN_BF16 ? few((const __bf16 *)x, ldx, w_codes, w_scales, n_rows, n_outputs, n_values, (__bf16 *)out, ldo, stream)
                              : few((const float *)x, ldx, w_codes, w_scales, n_rows, n_outputs, n_values, (float *)out, ldo, stream);
  }
  Carver c{(char *)workspace};
  uint8_t *codes = c.take<uint8_t>((size_t)(n_rows * blocks_of(n_values) * 16)), *scales = c.take<uint8_t>((size_t)(n_rows * blocks_of(n_values)));
  if ((st = sdnn_mx_quantize(x, ldx, dtype, n_rows, n_values, codes, scales, hip_stream)) != SDNN_OK) return st;
  return sdnn_mx_product(codes, scales, w_codes, w_scales, n_rows, n_outputs, n_values, out, ldo, dtype, hip_stream);
}

}  // extern "C"
