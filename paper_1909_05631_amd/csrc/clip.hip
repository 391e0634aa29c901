// The common norm of a list of tensors, n = sqrt(sum of v^2 over all of them), and the list scaled by min(1, most / n).
//
// The list is cut into pieces of one size, the list's 2048th part (a CU holds 8 workgroups, so 2048 run at once). Every
// tensor's last piece may be a shorter one: up to a tensor's number more pieces than 2048, which begin as others end (2077 for 240
// tensors of 77 MB). One launch for every 136 tensors (64 where one has rows apart from each other), whose descriptions travel
// as its arguments, leaves each piece's sum of squares and its description in the workspace; one more goes over all pieces: every
// workgroup sums the pieces' sums for itself, in the same order, and scales its piece. Neither waits for the host, and no
// sum depends on the order of arrival: the same list gives the same bits.
//
// Squares and sums are taken in 64 bits: a list's norm is exact to its rounding to fp32 whatever the values' sizes (squares of
// 1e-45 and of 3e38 are normal numbers there), and memory still bounds the pass.
// Bound by memory for large lists, which are read twice and written once: 16 tensors of 2.6 GB together 1.57 ms, 0.48 for the
// squares (5.3 TB/s) and 1.09 for the rest (4.7); a copy runs at 4.9. By launches and by the list's description for small ones: 3 of
// 4 MB together 17 us, of which the kernels take 8; 240 of 77 MB 138 us, 113 of them in the binding (64 us on the card).
#include "dense.h"

using namespace dense;

namespace {

constexpr int kMaxTensors = 4096, kPieces = 2048;
constexpr int64_t kLeastPiece = 8192, kUnit = 4096;  // bytes
constexpr int64_t kSegment = 4096;                   // bytes of a strided row that a workgroup takes by itself

// A run of values [start, start + count) of a matrix of `cols` columns; contiguous ones have one row.
struct Piece {
  const void *in;
  void *out;
  int64_t start, count, cols, ld, ldo;
  int dtype, contiguous;
};

// Tensors of one launch, and the first of each one's pieces there: contiguous ones, or any. (A launch's arguments stay
// below 4 KB.)
template <int COUNT>
struct List {
  static constexpr int kMost = COUNT;
  const void *in[COUNT];
  void *out[COUNT];
  int first[COUNT];
  int count, first_piece;  // tensors, and the launch's first piece
  int64_t bytes;           // of a piece
};
struct Contiguous : List<136> {
  int64_t size[136];  // values, twice, and one more for bf16
  __host__ void set(int i, int64_t, int64_t cols, int64_t, int64_t, int dtype) { size[i] = cols * 2 + (dtype == SDNN_BF16); }
  __device__ int dtype(int i) const { return size[i] & 1 ? SDNN_BF16 : SDNN_FP32; }
  __device__ Piece piece(int i, int64_t start, int64_t per) const {
    const int64_t all = size[i] >> 1;
    return {in[i], out[i], start, min(per, all - start), all, 0, 0, dtype(i), true};
  }
};
struct Strided : List<64> {
  int64_t rows[64], cols[64], ld[64], ldo[64];
  int8_t kind[64];
  __host__ void set(int i, int64_t r, int64_t c, int64_t l, int64_t lo, int dtype) {
    rows[i] = r;
    cols[i] = c;
    ld[i] = l;
    ldo[i] = lo;
    kind[i] = (int8_t)dtype;
  }
  __device__ int dtype(int i) const { return kind[i]; }
  __device__ Piece piece(int i, int64_t start, int64_t per) const {
    return {in[i], out[i], start, min(per, rows[i] * cols[i] - start), cols[i], ld[i], ldo[i], kind[i], rows[i] == 1};
  }
};
static_assert(sizeof(Contiguous) <= 4000 && sizeof(Strided) <= 4000, "a launch's arguments");

template <class T>
using Chunk = T __attribute__((ext_vector_type(16 / sizeof(T))));

// f(values) for 16 bytes of a contiguous run at a time, and for single values at its ends.
template <class T, class F, class G>
__device__ __forceinline__ void over_run(const T *p, int64_t n, const F &chunk, const G &single) {
  constexpr int N = 16 / sizeof(T);
  int64_t head = (int64_t)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T);
  if (head > n) head = n;
  if (threadIdx.x < head) single(threadIdx.x);
  const int64_t chunks = (n - head) / N;
#pragma unroll 4
  for (int64_t i = threadIdx.x; i < chunks; i += 256) chunk(head + i * N);
  const int64_t tail = head + chunks * N;
  if (threadIdx.x < n - tail) single(tail + threadIdx.x);
}

template <class T>
__device__ __forceinline__ double squares_of(const Piece &p) {
  double sum = 0.0;
  const auto add = [&](float v) { sum = fma((double)v, (double)v, sum); };
  const auto run = [&](const T *from, int64_t n) {
    over_run(from, n, [&](int64_t i) {
      const Chunk<T> v = *(const Chunk<T> *)(from + i);
#pragma unroll
      for (int e = 0; e < 16 / (int)sizeof(T); ++e) add((float)v[e]);
    }, [&](int64_t i) { add((float)from[i]); });
  };
  if (p.contiguous) {
    run((const T *)p.in + p.start, p.count);
  } else if (p.cols * (int64_t)sizeof(T) >= kSegment) {
    for (int64_t at = p.start, end = p.start + p.count; at < end;) {
      const int64_t r = at / p.cols, c = at - r * p.cols, n = min(p.cols - c, end - at);
      run((const T *)p.in + r * p.ld + c, n);
      at += n;
    }
  } else {
    for (int64_t i = threadIdx.x; i < p.count; i += 256) {
      const int64_t r = (p.start + i) / p.cols, c = p.start + i - r * p.cols;
      add((float)((const T *)p.in)[r * p.ld + c]);
    }
  }
  return sum;
}

// Sum over a workgroup of 256, in every thread.
__device__ __forceinline__ double sum_of_workgroup(double v) {
  __shared__ double part[4];
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

template <class L>
__global__ __launch_bounds__(256) void k_squares(const L list, Piece *pieces, double *sums) {
  const int lane = threadIdx.x & 63, b = blockIdx.x;
  // the last tensor whose pieces begin at or before this one
  int at = -1;
#pragma unroll
  for (int i = 0; i < L::kMost; i += 64) at += __popcll(__ballot(i + lane < list.count && list.first[min(i + lane, L::kMost - 1)] <= b));
  at = tile::uniform(at);
  const int dtype = list.dtype(at);
  const int64_t per = list.bytes / (dtype == SDNN_BF16 ? 2 : 4);
  const Piece p = list.piece(at, (b - list.first[at]) * per, per);
  const double sum = sum_of_workgroup(dtype == SDNN_BF16 ? squares_of<__bf16>(p) : squares_of<float>(p));
  if (threadIdx.x == 0) {
    pieces[list.first_piece + b] = p;
    sums[list.first_piece + b] = sum;
  }
}

__device__ __forceinline__ double norm_of(const double *sums, int count) {
  double v = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < count; i += 256) v += sums[i];
  return sqrt(sum_of_workgroup(v));
}

__global__ __launch_bounds__(256) void k_norm(const double *sums, int count, float *norm) {
  const double n = norm_of(sums, count);
  if (threadIdx.x == 0) *norm = (float)n;
}

template <class T>
__device__ __forceinline__ void scale_piece(const Piece &p, float by) {
  const auto run = [&](const T *from, T *to, int64_t n) {
    if ((((uintptr_t)from ^ (uintptr_t)to) & 15) == 0) {
      over_run(from, n, [&](int64_t i) {
        Chunk<T> v = *(const Chunk<T> *)(from + i);
#pragma unroll
        for (int e = 0; e < 16 / (int)sizeof(T); ++e) v[e] = (T)((float)v[e] * by);
        *(Chunk<T> *)(to + i) = v;
      }, [&](int64_t i) { to[i] = (T)((float)from[i] * by); });
    } else {
#pragma unroll 4
      for (int64_t i = threadIdx.x; i < n; i += 256) to[i] = (T)((float)from[i] * by);
    }
  };
  if (p.contiguous) {
    run((const T *)p.in + p.start, (T *)p.out + p.start, p.count);
  } else if (p.cols * (int64_t)sizeof(T) >= kSegment) {
    for (int64_t at = p.start, end = p.start + p.count; at < end;) {
      const int64_t r = at / p.cols, c = at - r * p.cols, n = min(p.cols - c, end - at);
      run((const T *)p.in + r * p.ld + c, (T *)p.out + r * p.ldo + c, n);
      at += n;
    }
  } else {
    for (int64_t i = threadIdx.x; i < p.count; i += 256) {
      const int64_t r = (p.start + i) / p.cols, c = p.start + i - r * p.cols;
      ((T *)p.out)[r * p.ldo + c] = (T)((float)((const T *)p.in)[r * p.ld + c] * by);
    }
  }
}

// A norm past `most`, or one that is NaN, scales; an infinite one leaves zeros (and NaN of what was infinite).
__global__ __launch_bounds__(256) void k_clip(const Piece *pieces, const double *sums, int count, float most, float *norm) {
  const double n = norm_of(sums, count);
  if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)n;
  const float by = n <= (double)most ? 1.0f : (float)((double)most / n);
  const Piece p = pieces[blockIdx.x];
  if (by == 1.0f && p.in == p.out) return;
  if (p.dtype == SDNN_BF16)
    scale_piece<__bf16>(p, by);
  else
    scale_piece<float>(p, by);
}

// ------------------------------------------------------------------------------------------------
// Host

struct Space {
  Piece *pieces;
  double *sums;
  Space(Carver &c, int64_t n) {
    pieces = c.take<Piece>((size_t)(kPieces + n));
    sums = c.take<double>((size_t)(kPieces + n));
  }
};

// Two tensors that are written to one place would be scaled twice; which of the two results stayed would be chance.
bool all_apart(const sdnn_tensor *tensors, int n, bool clip, int *first, int *second) {
  constexpr int kSlots = 2 * kMaxTensors;
  uint16_t slot[kSlots];  // index + 1
  int mask = 16;
  while (mask < 2 * n) mask *= 2;
  for (int i = 0; i < mask; ++i) slot[i] = 0;
  --mask;
  for (int i = 0; i < n; ++i) {
    if (!clip || tensors[i].rows == 0 || tensors[i].cols == 0) continue;
    const void *to = tensors[i].out ? tensors[i].out : tensors[i].data;
    uint64_t at = ((uint64_t)(uintptr_t)to >> 1) * 0x9e3779b97f4a7c15ull >> 40;
    for (;; ++at) {
      const int j = slot[at & mask];
      if (j == 0) break;
      const void *other = tensors[j - 1].out ? tensors[j - 1].out : tensors[j - 1].data;
      if (other == to) {
        *first = j - 1;
        *second = i;
        return false;
      }
    }
    slot[at & mask] = (uint16_t)(i + 1);
  }
  return true;
}

sdnn_status check_list(const sdnn_tensor *tensors, int64_t n, bool clip) {
  if (n < 0 || n > kMaxTensors) return fail(SDNN_EINVAL, "n_tensors %lld is outside [0, %d]", (long long)n, kMaxTensors);
  if (n && !tensors) return fail(SDNN_EINVAL, "tensors is null");
  for (int64_t i = 0; i < n; ++i) {
    const sdnn_tensor &t = tensors[i];
    if (!good_dtype(t.dtype)) return fail(SDNN_EINVAL, "tensor %lld: dtype %d is neither SDNN_FP32 nor SDNN_BF16", (long long)i, t.dtype);
    if (t.rows < 0 || t.cols < 0 || t.rows > 1ll << 40 || t.cols > 1ll << 40 || (t.cols && t.rows > (1ll << 40) / t.cols))
      return fail(SDNN_EINVAL, "tensor %lld: %lld x %lld values are outside [0, 2^40]", (long long)i, (long long)t.rows, (long long)t.cols);
    if (t.rows == 0 || t.cols == 0) continue;
    if (!t.data || (uintptr_t)t.data % dtype_bytes(t.dtype)) return fail(SDNN_EINVAL, "tensor %lld: data is null or not aligned to its values", (long long)i);
    if (t.rows > 1 && (t.ld < t.cols || t.ld > 1ll << 40)) return fail(SDNN_EINVAL, "tensor %lld: the row stride %lld is outside [%lld, 2^40]", (long long)i, (long long)t.ld, (long long)t.cols);
    if (!clip) continue;
    if ((uintptr_t)t.out % dtype_bytes(t.dtype)) return fail(SDNN_EINVAL, "tensor %lld: out is not aligned to its values", (long long)i);
    if (t.out && t.rows > 1 && (t.ldo < t.cols || t.ldo > 1ll << 40)) return fail(SDNN_EINVAL, "tensor %lld: the row stride of out, %lld, is outside [%lld, 2^40]", (long long)i, (long long)t.ldo, (long long)t.cols);
    if (t.out == t.data && t.rows > 1 && t.ldo != t.ld) return fail(SDNN_EINVAL, "tensor %lld: out is data with another row stride", (long long)i);
  }
  int a, b;
  if (!all_apart(tensors, (int)n, clip, &a, &b)) return fail(SDNN_EINVAL, "tensors %d and %d are written to the same place", a, b);
  return SDNN_OK;
}

// The pieces' sums and descriptions; `total` of them.
bool contiguous(const sdnn_tensor &t) { return t.rows <= 1 || (t.ld == t.cols && (!t.out || t.ldo == t.cols)); }

template <class L>
sdnn_status squares_of_list(const sdnn_tensor *tensors, int64_t n, int64_t piece, const Space &sp, int *total, hipStream_t stream) {
  L list;
  list.bytes = piece;
  list.count = list.first_piece = 0;
  int here = 0;  // pieces of this launch
  for (int64_t i = 0; i < n; ++i) {
    const sdnn_tensor &t = tensors[i];
    const int64_t size = t.rows * t.cols * dtype_bytes(t.dtype);
    if (size > 0) {
      const int k = list.count++;
      const bool flat = contiguous(t);
      list.in[k] = t.data;
      list.out[k] = t.out ? t.out : t.data;
      list.first[k] = here;
      list.set(k, flat ? 1 : t.rows, flat ? t.rows * t.cols : t.cols, t.ld, t.out ? t.ldo : t.ld, t.dtype);
      here += (int)ceil_div(size, piece);
    }
    if (list.count == L::kMost || (i == n - 1 && list.count > 0)) {
      hipLaunchKernelGGL((k_squares<L>), dim3((unsigned)here), dim3(256), 0, stream, list, sp.pieces, sp.sums);
      const sdnn_status st = launched("squares");
      if (st != SDNN_OK) return st;
      list.first_piece += here;
      list.count = here = 0;
    }
  }
  *total = list.first_piece;
  return SDNN_OK;
}

sdnn_status squares(const sdnn_tensor *tensors, int64_t n, const Space &sp, int *total, hipStream_t stream) {
  int64_t bytes = 0;
  bool flat = true;
  for (int64_t i = 0; i < n; ++i) {
    bytes += tensors[i].rows * tensors[i].cols * dtype_bytes(tensors[i].dtype);
    flat = flat && contiguous(tensors[i]);
  }
  const int64_t piece = std::max(kLeastPiece, ceil_div(ceil_div(bytes, kPieces), kUnit) * kUnit);
  return flat ? squares_of_list<Contiguous>(tensors, n, piece, sp, total, stream) : squares_of_list<Strided>(tensors, n, piece, sp, total, stream);
}

}  // namespace

extern "C" {

size_t sdnn_clip_workspace_bytes(int64_t n_tensors) {
  if (n_tensors < 0 || n_tensors > kMaxTensors) return 0;
  Carver c{nullptr};
  Space s(c, n_tensors);
  return c.used;
}

sdnn_status sdnn_global_norm(const sdnn_tensor *tensors, int64_t n_tensors, float *norm, void *workspace, size_t workspace_bytes, void *hip_stream) {
  sdnn_status st = check_list(tensors, n_tensors, false);
  if (st != SDNN_OK) return st;
  if (!norm || (uintptr_t)norm % 4) return fail(SDNN_EINVAL, "norm is null or not aligned");
  if ((st = check_workspace(workspace, workspace_bytes, sdnn_clip_workspace_bytes(n_tensors))) != SDNN_OK) return st;
  Carver c{(char *)workspace};
  const Space sp(c, n_tensors);
  int total;
  if ((st = squares(tensors, n_tensors, sp, &total, (hipStream_t)hip_stream)) != SDNN_OK) return st;
  hipLaunchKernelGGL(k_norm, dim3(1), dim3(256), 0, (hipStream_t)hip_stream, sp.sums, total, norm);
  return launched("norm");
}

sdnn_status sdnn_clip(const sdnn_tensor *tensors, int64_t n_tensors, float max_norm, float *norm, void *workspace, size_t workspace_bytes, void *hip_stream) {
  sdnn_status st = check_list(tensors, n_tensors, true);
  if (st != SDNN_OK) return st;
  if (!(max_norm >= 0.0f)) return fail(SDNN_EINVAL, "max_norm %g is not at least 0", max_norm);
  if (!norm || (uintptr_t)norm % 4) return fail(SDNN_EINVAL, "norm is null or not aligned");
  if ((st = check_workspace(workspace, workspace_bytes, sdnn_clip_workspace_bytes(n_tensors))) != SDNN_OK) return st;
  Carver c{(char *)workspace};
  const Space sp(c, n_tensors);
  int total;
  if ((st = squares(tensors, n_tensors, sp, &total, (hipStream_t)hip_stream)) != SDNN_OK) return st;
  if (total > 0)
    hipLaunchKernelGGL(k_clip, dim3((unsigned)total), dim3(256), 0, (hipStream_t)hip_stream, sp.pieces, sp.sums, total, max_norm, norm);
  else
    hipLaunchKernelGGL(k_norm, dim3(1), dim3(256), 0, (hipStream_t)hip_stream, sp.sums, 0, norm);
  return launched("clip");
}

}  // extern "C"
