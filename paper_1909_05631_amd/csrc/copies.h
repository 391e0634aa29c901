// Operands that are written anew before a tile product: up to three matrices of as many columns in one launch.
#ifndef SDNN_COPIES_H
#define SDNN_COPIES_H

#include "dense.h"
#include "few.h"

namespace copies {

using namespace dense;

// A matrix and where its rows go: fp32 in two fp16 parts under a power of two a row, in three bf16 parts, or as they are on
// aligned rows.
struct Source {
  const void *data;
  int64_t ld, rows;
  char *out;
  int *exponents;  // of two parts
  bool vec;
};
struct Sources {
  Source of[3];
  int64_t cols;
};

// The source that row r of all of them is of, and its row there.
__device__ __forceinline__ const Source &source_of(const Sources &s, int64_t &r) {
  int i = 0;
  while (i < 2 && r >= s.of[i].rows) r -= s.of[i++].rows;
  return s.of[i];
}

// Two parts, zeros past the columns, a workgroup a row.
[[maybe_unused]] static __global__ __launch_bounds__(256) void k_two_parts(Sources s, int64_t rows) {
  __shared__ float part[4];
  const int64_t groups = ceil_div(s.cols, 32);
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x) {
    int64_t r = i;
    const Source &m = source_of(s, r);
    const float *row = (const float *)m.data + r * m.ld;
    float top = 0.0f;
    for (int64_t k = threadIdx.x * 4; k < s.cols; k += 1024) {
      const f32x4 v = few::load4(row, (int)k, (int)s.cols, m.vec);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float a = fabsf(v[e]);
        top = fmaxf(top, a < __builtin_inff() ? a : 0.0f);  // infinities and NaN have no say
      }
    }
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = top;
    __syncthreads();
    const int e = split_exponent(fmaxf(fmaxf(part[0], part[1]), fmaxf(part[2], part[3])));
    if (threadIdx.x == 0) m.exponents[r] = e;
    char *to = m.out + r * groups * 128;
    for (int64_t k = threadIdx.x * 4; k < groups * 32; k += 1024) {
      f32x4 v = few::load4(row, (int)k, (int)s.cols, m.vec);
#pragma unroll
      for (int c = 0; c < 4; ++c) v[c] = ldexpf(v[c], e);
      store_split4(to, k, v);
    }
  }
}

// Three parts, zeros past the columns.
[[maybe_unused]] static __global__ __launch_bounds__(256) void k_three_parts(Sources s, int64_t rows) {
  const int64_t groups = ceil_div(s.cols, 64);
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x) {
    int64_t r = i;
    const Source &m = source_of(s, r);
    const float *row = (const float *)m.data + r * m.ld;
    char *to = m.out + r * groups * tile::kGroup3;
    for (int64_t k = threadIdx.x * 4; k < groups * 64; k += 1024) store_three4(to, k, few::load4(row, (int)k, (int)s.cols, m.vec));
  }
}

// On rows of whole 16 bytes, zeros past the columns.
template <class T>
__global__ __launch_bounds__(256) void k_aligned(Sources s, int64_t rows) {
  const int64_t pitch = ceil_div(s.cols, 8) * 8;
  for (int64_t i = blockIdx.x; i < rows; i += gridDim.x) {
    int64_t r = i;
    const Source &m = source_of(s, r);
    const T *row = (const T *)m.data + r * m.ld;
    T *to = (T *)m.out + r * pitch;
    for (int64_t k = threadIdx.x * 4; k < pitch; k += 1024) store4(to + k, few::load4(row, (int)k, (int)s.cols, m.vec), 4, true);
  }
}

}  // namespace copies

#endif  // SDNN_COPIES_H
