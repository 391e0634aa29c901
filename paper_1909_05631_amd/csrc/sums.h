// What readout.hip and its neighbours share around the tile products: storing sums, joining those of a split k, and what a
// matrix's rows are aligned for.
#ifndef SDNN_SUMS_H
#define SDNN_SUMS_H

#include "dense.h"

namespace sums {

using namespace dense;

// Sums stored in the output's type.
template <class T>
struct Store {
  using Value = T;
  T *out;
  int64_t ld, rows, cols;
  bool vec;
  const float *factor = nullptr;  // what the sums are multiplied by: the mean's, or the heaviest weight
  const float *before = nullptr;  // sums of the pieces before
  int64_t ld_before = 0;
  __device__ __forceinline__ T *row(int64_t r) const { return out + r * ld; }  // r < rows
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

// The slabs' sum, rounded to the output's type: 256 / GROUPS items a workgroup, each group taking every GROUPS-th slab. S: a
// Store, or another that says where a row goes (nullptr: nowhere).
template <class S, int GROUPS>
__global__ __launch_bounds__(256) void k_sum_slabs(const float *slabs, int splits, int64_t ld_slab, S to) {
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
    if (group == 0 && i < total && c < to.cols) {
      typename S::Value *out = to.row(r);
      if (out) store4(out + c, v * by, (int)(to.cols - c < 4 ? to.cols - c : 4), to.vec);
    }
  }
}

template <class S>
sdnn_status sum_slabs(const float *slabs, int splits, int64_t ld_slab, const S &to, hipStream_t stream, const char *what) {
  const int64_t items = to.rows * (ld_slab / 4);
  if (splits >= 32)
    hipLaunchKernelGGL((k_sum_slabs<S, 16>), dim3((unsigned)std::min<int64_t>(ceil_div(items, 16), 8192)), dim3(256), 0, stream, slabs, splits, ld_slab, to);
  else if (splits >= 8)
    hipLaunchKernelGGL((k_sum_slabs<S, 4>), dim3((unsigned)std::min<int64_t>(ceil_div(items, 64), 8192)), dim3(256), 0, stream, slabs, splits, ld_slab, to);
  else
    hipLaunchKernelGGL((k_sum_slabs<S, 1>), dim3((unsigned)std::min<int64_t>(ceil_div(items, 256), 8192)), dim3(256), 0, stream, slabs, splits, ld_slab, to);
  return launched(what);
}

// Rows that the tiles read as they are: whole dwords.
inline bool usable_in_place(const void *p, int64_t ld, int64_t cols, int bytes) {
  return ((uintptr_t)p & 3) == 0 && ld * bytes % 4 == 0 && cols * bytes % 4 == 0 && ld * bytes <= kMaxPitch;
}

inline unsigned row_grid(int64_t rows) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>(rows, 2048)); }

inline bool aligned16(const void *p, int64_t ld, int bytes) { return ((uintptr_t)p & 15) == 0 && ld * bytes % 16 == 0; }

template <class T>
bool vector_rows(const T *p, int64_t ld) {  // aligned for 16 bytes
  return (uintptr_t)p % 16 == 0 && ld * sizeof(T) % 16 == 0;
}

}  // namespace sums

#endif  // SDNN_SUMS_H
