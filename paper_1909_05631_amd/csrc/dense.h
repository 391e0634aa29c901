// What the dense operators (readout.hip, orthogonalize.hip, mx.hip) share around tile.h: checks of arguments, the
// order of blocks, split sums, storing.
#ifndef SDNN_DENSE_H
#define SDNN_DENSE_H

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "error.h"
#include "tile.h"

namespace dense {

using tile::f32x4;

constexpr int kXcds = 8;
constexpr int kCus = 256;  // compute units: what a launch has to fill
constexpr int64_t kMaxRows = 1 << 24, kMaxClasses = 1 << 24, kMaxFeatures = 1 << 20;
constexpr int64_t kMaxPitch = 1 << 22;  // bytes from row to row that the tiles' 32-bit offsets reach over 256 rows

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int64_t ceil_div(int64_t x, int64_t a) { return (x + a - 1) / a; }

inline bool good_dtype(int32_t d) { return d == SDNN_FP32 || d == SDNN_BF16; }
inline int dtype_bytes(int32_t d) { return d == SDNN_BF16 ? 2 : 4; }

// A kernel's launch reported as a status.
inline sdnn_status launched(const char *what) {
  const hipError_t e = hipGetLastError();
  return e == hipSuccess ? SDNN_OK : fail(SDNN_EDEVICE, "%s: %s", what, hipGetErrorString(e));
}

// The workspace as consecutive 256-byte aligned parts; with base == nullptr it only counts.
struct Carver {
  char *base;
  size_t used = 0;
  template <class T>
  T *take(size_t count) {
    T *p = base ? reinterpret_cast<T *>(base + used) : nullptr;
    used += align_up(count * sizeof(T), 256);
    return p;
  }
};

__device__ __forceinline__ float load_as_float(const float *p) { return *p; }
__device__ __forceinline__ float load_as_float(const __bf16 *p) { return (float)*p; }

// Four neighbours of one row; `vec`: the row is aligned for one store. The rounding to bf16 is the output's own.
__device__ __forceinline__ void store4(float *p, f32x4 v, int n, bool vec) {
  if (vec && n >= 4) {
    *(f32x4 *)p = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = v[i];
  }
}
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ void store4(__bf16 *p, f32x4 v, int n, bool vec) {
  const bf16x4 b = __builtin_convertvector(v, bf16x4);
  if (vec && n >= 4) {
    *(bf16x4 *)p = b;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) p[i] = b[i];
  }
}

// Where value k of a row lies in the split form: groups of 32 values, 64 bytes of high parts, 64 of low ones.
__device__ __forceinline__ int64_t split_at(int64_t k) { return (k >> 5) * 128 + (k & 31) * 2; }
constexpr int kLow = 64;

// v as high + low. A high part that is not finite has a zero low part (inf - inf would make a NaN of it).
__device__ __forceinline__ void split(float v, _Float16 &hi, _Float16 &lo) {
  hi = (_Float16)v;
  const float r = v - (float)hi;
  lo = __builtin_isfinite(r) ? (_Float16)r : (_Float16)0.0f;
}
__device__ __forceinline__ void store_split4(char *row, int64_t k, f32x4 v) {
  f16x4 hi, lo;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    _Float16 h, l;
    split(v[i], h, l);
    hi[i] = h;
    lo[i] = l;
  }
  *(f16x4 *)(row + split_at(k)) = hi;
  *(f16x4 *)(row + split_at(k) + kLow) = lo;
}

// The power of two that takes a largest magnitude to [2^14, 2^15), as an exponent: high parts stay finite in
// fp16 and values down to 2^-17 of the largest keep all their bits.
__device__ __forceinline__ int split_exponent(float top) {
  return top > 0.0f && top < __builtin_inff() ? 14 - ilogbf(top) : 0;
}

// Outputs of a launch in blocks. Workgroup ids go round the XCDs, so each XCD gets a run of consecutive
// blocks, and those go down 8 blocks of rows before the next column: an XCD's 32 CUs work on 8 x 4 blocks,
// which share their operands in its L2.
struct Blocks {
  int rows, cols, splits;  // blocks of rows, of columns, parts of k
  int64_t slabs;           // of all of k
  __device__ __forceinline__ void locate(int id, int total, int &r, int &c, int &split) const {
    const int whole = total / kXcds * kXcds;
    if (id < whole) id = id % kXcds * (total / kXcds) + id / kXcds;
    const int per = rows * cols;
    split = id / per;
    id -= split * per;
    const int tall = 8 * cols, g = id / tall, in = id - g * tall;
    const int h = rows - g * 8 < 8 ? rows - g * 8 : 8;
    c = in / h;
    r = g * 8 + in - c * h;
  }
  __device__ __forceinline__ void range(int split, int64_t &s0, int64_t &s1) const {
    const int64_t per = (slabs + splits - 1) / splits;
    s0 = split * per < slabs ? split * per : slabs;
    s1 = s0 + per < slabs ? s0 + per : slabs;
  }
};

// An operand of a whole launch; `at` gives the part of one block.
struct Matrix {
  const char *data;
  int64_t pitch;   // bytes
  int64_t rows;    // along: rows; across: rows of k
  int64_t extent;  // bytes in a row: of k (along), of columns (across)
  template <int KIND, int SIZE, bool ACROSS>
  __device__ __forceinline__ tile::Operand at(int block) const {
    const int64_t first = (int64_t)block * SIZE;
    if (ACROSS) {
      const int64_t skip = first * tile::Geometry<KIND>::kBytes;
      return {data + skip, pitch, rows, extent - skip};
    }
    return {data + first * pitch, pitch, rows - first, extent};
  }
};

template <class B, int KIND, int BM, int BN, bool ACROSS_A, bool ACROSS_B, class Epilogue>
__global__ __launch_bounds__(B::kThreads) void k_product(Matrix a, Matrix b, Blocks blocks, Epilogue epilogue) {
  __shared__ __attribute__((aligned(1024))) char lds[B::kLds];
  int r, c, split;
  blocks.locate(blockIdx.x, gridDim.x, r, c, split);
  int64_t s0, s1;
  blocks.range(split, s0, s1);
  B block;
  block.run(a.template at<KIND, BM, ACROSS_A>(r), b.template at<KIND, BN, ACROSS_B>(c), s0, s1, lds);
  epilogue(block, (int64_t)r * BM + B::row0(), (int64_t)c * BN + B::col0(), split, c);
}

// Launches the blocks of one shape. What the sizes need of it is the caller's rule.
template <int KIND, int BM, int BN, int WM, int WN, bool ACROSS_A, bool ACROSS_B, class Epilogue>
sdnn_status launch(const Matrix &a, const Matrix &b, int64_t rows, int64_t cols, int64_t k, int splits, const Epilogue &e, hipStream_t stream, const char *what) {
  using B = tile::Block<KIND, BM, BN, WM, WN, ACROSS_A, ACROSS_B>;
  Blocks blocks;
  blocks.slabs = ceil_div(k, tile::Geometry<KIND>::kPerSlab);
  blocks.splits = splits;
  const int64_t r = ceil_div(rows, BM), c = ceil_div(cols, BN);
  if (r * c * splits * B::kThreads > 0xffffffffll || a.pitch > kMaxPitch || b.pitch > kMaxPitch) return fail(SDNN_EINVAL, "%s: %lld x %lld outputs are too many for one launch", what, (long long)rows, (long long)cols);
  blocks.rows = (int)r;
  blocks.cols = (int)c;
  hipLaunchKernelGGL((k_product<B, KIND, BM, BN, ACROSS_A, ACROSS_B, Epilogue>), dim3((unsigned)(r * c * splits)), dim3(B::kThreads), 0, stream, a, b, blocks, e);
  return launched(what);
}

}  // namespace dense

#endif  // SDNN_DENSE_H
