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

// The slabs' sum, rounded to the output's type: THREADS / GROUPS items a workgroup, each group taking every GROUPS-th slab. S:
// a Store, or another that says where a row goes (nullptr: nowhere). `shared`: an f32x4 a thread.
template <class S, int GROUPS>
__device__ __forceinline__ void sum_of_slabs(const float *slabs, int splits, int64_t ld_slab, const S &to, int block, int blocks, int threads, f32x4 *shared) {
  const int items = threads / GROUPS;
  const int64_t per = ld_slab / 4, total = to.rows * per;
  const float by = to.factor ? *to.factor : 1.0f;
  const int group = threadIdx.x / items, item = threadIdx.x % items;
  for (int64_t i0 = (int64_t)block * items; i0 < total; i0 += (int64_t)blocks * items) {
    const int64_t i = i0 + item, r = i / per, c = (i - r * per) * 4;
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (i < total)
#pragma unroll 8
      for (int s = group; s < splits; s += GROUPS) v += *(const f32x4 *)(slabs + (s * to.rows + r) * ld_slab + c);
    if constexpr (GROUPS > 1) {
      __syncthreads();
      shared[threadIdx.x] = v;
      __syncthreads();
      if (group == 0)
        for (int g = 1; g < GROUPS; ++g) v += shared[g * items + item];
    }
    if (group == 0 && i < total && c < to.cols) {
      typename S::Value *out = to.row(r);
      if (out) store4(out + c, v * by, (int)(to.cols - c < 4 ? to.cols - c : 4), to.vec);
    }
  }
}
template <class S, int GROUPS>
__global__ __launch_bounds__(256) void k_sum_slabs(const float *slabs, int splits, int64_t ld_slab, S to) {
  __shared__ f32x4 shared[256];
  sum_of_slabs<S, GROUPS>(slabs, splits, ld_slab, to, blockIdx.x, gridDim.x, 256, shared);
}
inline int sum_groups(int splits) { return splits >= 32 ? 16 : splits >= 8 ? 4 : 1; }

template <class S>
sdnn_status sum_slabs(const float *slabs, int splits, int64_t ld_slab, const S &to, hipStream_t stream, const char *what) {
  const int64_t items = to.rows * (ld_slab / 4);
  const int groups = sum_groups(splits);
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(items, 256 / groups), 8192));
  if (groups == 16)
    hipLaunchKernelGGL((k_sum_slabs<S, 16>), grid, dim3(256), 0, stream, slabs, splits, ld_slab, to);
  else if (groups == 4)
    hipLaunchKernelGGL((k_sum_slabs<S, 4>), grid, dim3(256), 0, stream, slabs, splits, ld_slab, to);
  else
    hipLaunchKernelGGL((k_sum_slabs<S, 1>), grid, dim3(256), 0, stream, slabs, splits, ld_slab, to);
  return launched(what);
}

// The same by the last workgroups of the next product's launch, for one launch less (none: count is 0).
template <class S>
struct SumTail {
  static constexpr bool kAny = true;
  const float *slabs;
  int splits, count, groups;
  int64_t ld_slab;
  S to;
  __host__ __device__ int blocks() const { return count; }
  __device__ __forceinline__ void operator()(int block, int threads, char *lds) const {
    if (groups == 16)
      sum_of_slabs<S, 16>(slabs, splits, ld_slab, to, block, count, threads, (f32x4 *)lds);
    else if (groups == 4)
      sum_of_slabs<S, 4>(slabs, splits, ld_slab, to, block, count, threads, (f32x4 *)lds);
    else
      sum_of_slabs<S, 1>(slabs, splits, ld_slab, to, block, count, threads, (f32x4 *)lds);
  }
};
template <class S>
SumTail<S> sum_tail(const float *slabs, int splits, int64_t ld_slab, const S &to) {
  const int groups = sum_groups(splits);
  const int64_t items = to.rows * (ld_slab / 4);
  return {slabs, splits, (int)std::min<int64_t>(ceil_div(items, 256 / groups), 1024), groups, ld_slab, to};
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
