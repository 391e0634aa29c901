// What the dense operators (readout.hip, orthogonalize.hip, mx.hip) share around tile.h: checks of arguments, the
// order of blocks, split sums, storing.
#ifndef SDNN_DENSE_H
#define SDNN_DENSE_H

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "error.h"
#include "tile.h"

namespace dense {

using sdnn_error::fail;
using tile::f32x4;

constexpr int kXcds = 8;
constexpr int kCus = 256;  // compute units: what a launch has to fill
constexpr int64_t kMaxRows = 1 << 24, kMaxClasses = 1 << 24, kMaxFeatures = 1 << 20;
constexpr int kMaxSplits = 64;
constexpr int64_t kMaxPitch = 6 << 20;  // bytes from row to row: the longest row in three parts; the tiles' 32-bit offsets reach over 256 rows

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
__host__ __device__ inline int64_t ceil_div(int64_t x, int64_t a) { return (x + a - 1) / a; }

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

// A subtile row of a block's results, columns [col, col + 16 * N) of row `to`, by the four lane groups that hold it: for
// bf16 neighbouring groups exchange halves of two subtiles, so that a lane stores 16 bytes.
template <class T, int N, class F>
__device__ __forceinline__ void store_row(T *to, int64_t col, int64_t cols, bool vec, bool in, const F &value) {
  const int j4 = (threadIdx.x & 63) >> 4;
  if constexpr (sizeof(T) == 2 && N % 2 == 0) {
#pragma unroll
    for (int j = 0; j < N; j += 2) {
      typedef int i32x2 __attribute__((ext_vector_type(2)));
      typedef int i32x4 __attribute__((ext_vector_type(4)));
      const i32x2 a = __builtin_bit_cast(i32x2, __builtin_convertvector(value(j), bf16x4)), b = __builtin_bit_cast(i32x2, __builtin_convertvector(value(j + 1), bf16x4));
      const bool odd = j4 & 1;  // even groups take subtile j's 8 columns from 4 j4 on, odd ones subtile j + 1's from 4 (j4 - 1) on
      i32x2 pass, own, got;
      pass[0] = odd ? a[0] : b[0];
      pass[1] = odd ? a[1] : b[1];
      own[0] = odd ? b[0] : a[0];
      own[1] = odd ? b[1] : a[1];
      got[0] = __shfl_xor(pass[0], 16);
      got[1] = __shfl_xor(pass[1], 16);
      const int64_t c = col + 16 * (j + odd) + 4 * (j4 & 2);
      const i32x4 both = odd ? i32x4{got[0], got[1], own[0], own[1]} : i32x4{own[0], own[1], got[0], got[1]};
      if (in && c < cols) {
        if (vec && c + 8 <= cols) {
          *(i32x4 *)(to + c) = both;
        } else {
          typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
          const bf16x8 v = __builtin_bit_cast(bf16x8, both);
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (c + i < cols) to[c + i] = v[i];
        }
      }
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const int64_t c = col + 16 * j + 4 * j4;
      const f32x4 v = value(j);
      if (in && c < cols) store4(to + c, v, (int)(cols - c < 4 ? cols - c : 4), vec);
    }
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

// v as high + middle + low in bf16, exactly (while low stays normal); a value past bf16's largest has its high part cut, not
// rounded to infinity.
__device__ __forceinline__ void split3(float v, __bf16 &hi, __bf16 &mid, __bf16 &lo) {
  hi = (__bf16)v;
  if (!__builtin_isfinite((float)hi) && __builtin_isfinite(v)) hi = (__bf16)__uint_as_float(__float_as_uint(v) & 0xffff0000u);
  const float r = __builtin_isfinite((float)hi) ? v - (float)hi : 0.0f;
  mid = (__bf16)r;
  lo = (__bf16)(r - (float)mid);
}
// Four neighbours of a row in the form of KIND_THREE.
__device__ __forceinline__ void store_three4(char *row, int64_t k, f32x4 v) {
  bf16x4 hi, mid, lo;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __bf16 h, m, l;
    split3(v[i], h, m, l);
    hi[i] = h;
    mid[i] = m;
    lo[i] = l;
  }
  char *to = row + (k >> 6) * tile::kGroup3 + (k & 63) * 2;
  *(bf16x4 *)to = hi;
  *(bf16x4 *)(to + tile::kSlab) = mid;
  *(bf16x4 *)(to + 2 * tile::kSlab) = lo;
}

// The power of two that takes a largest magnitude to [2^14, 2^15), as an exponent: high parts stay finite in
// fp16 and values down to 2^-17 of the largest keep all their bits.
__device__ __forceinline__ int split_exponent(float top) {
  return top > 0.0f && top < __builtin_inff() ? 14 - ilogbf(top) : 0;
}

// Sums kept in fp32, one slab per part of k (and matrix of a batch); with `add`, on what is there already.
struct Accumulate {
  float *slabs;
  int64_t ld, rows, cols;
  bool add;
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int split, bool) const {
    const int lane = threadIdx.x & 63, i16 = lane & 15, j4 = lane >> 4;
    float *slab = slabs + ((int64_t)split * gridDim.y + blockIdx.y) * rows * ld;
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

// Outputs of a launch in blocks. Workgroup ids go round the XCDs, so each XCD gets a run of consecutive
// blocks, and those go down 8 blocks of rows before the next column: an XCD's 32 CUs work on 8 x 4 blocks,
// which share their operands in its L2.
struct Blocks {
  int rows, cols, splits;  // blocks of rows, of columns, parts of k
  int slabs, per;          // slabs of all of k, of a part
  bool symmetric;          // square blocks on and above the diagonal only
  __device__ __forceinline__ void locate(int id, int total, int &r, int &c, int &split) const {
    const int whole = total / kXcds * kXcds;
    if (id < whole) id = id % kXcds * (total / kXcds) + id / kXcds;
    if (symmetric) {
      c = (int)((sqrtf(8.0f * id + 1.0f) - 1.0f) * 0.5f);
      while (c * (c + 1) / 2 > id) --c;
      while ((c + 1) * (c + 2) / 2 <= id) ++c;
      r = id - c * (c + 1) / 2;
      split = 0;
      return;
    }
    const int area = rows * cols;
    split = id / area;
    id -= split * area;
    const int tall = 8 * cols, g = id / tall, in = id - g * tall;
    const int h = rows - g * 8 < 8 ? rows - g * 8 : 8;
    c = in / h;
    r = g * 8 + in - c * h;
  }
  __device__ __forceinline__ void range(int split, int &s0, int &s1) const {
    s0 = tile::uniform(min(split * per, slabs));
    s1 = tile::uniform(min(s0 + per, slabs));
  }
};

// An operand of a whole launch; `at` gives the part of one block.
struct Matrix {
  const char *data;
  int64_t pitch;   // bytes
  int64_t rows;    // along: rows; across: rows of k
  int64_t extent;  // bytes in a row: of k (along), of columns (across); KIND_THREE: of one part
  int64_t batch;   // bytes from one matrix of a batch (blockIdx.y) to the next
  const uint8_t *scales = nullptr;  // KIND_MX: pitch / 16 bytes a row
  // An operand of two matrices of `rows` rows each (tile::Operand). across: the first's rows of k are padded to `units` slabs
  const char *second = nullptr;
  int64_t pitch_second = 0;
  int units = 0;
  template <int KIND, int SIZE, bool ACROSS, bool TWO = false>
  __device__ __forceinline__ tile::Operand at(int block) const {
    if constexpr (TWO) {
      constexpr int kRows = tile::Geometry<KIND>::kPerSlab;  // of k in a slab across
      tile::Operand o = at<KIND, ACROSS ? SIZE : SIZE / 2, ACROSS>(block);
      const int64_t first = (int64_t)block * (SIZE / 2);  // along: of each
      const int64_t skip = ACROSS ? o.base - data : first * pitch_second;
      o.second = second + skip;
      o.pitch_second = (int)pitch_second;
      if (ACROSS) {
        o.units = units;
        o.first_rows = (int)rows;
        o.rows = (int)(units * kRows + rows);
      }
      return o;
    }
    const int64_t first = (int64_t)block * SIZE;
    const char *here = data + blockIdx.y * batch;
    if (ACROSS && KIND == tile::KIND_THREE) {
      const int64_t group = first / 64;
      return {here + group * tile::kGroup3, (int)pitch, (int)rows, (int)(extent - group * tile::kSlab), nullptr, (int)(first % 64) * 2};
    }
    if (ACROSS) {
      const int64_t skip = first * tile::Geometry<KIND>::kBytes;
      return {here + skip, (int)pitch, (int)rows, (int)(extent - skip)};
    }
    return {here + first * pitch, (int)pitch, (int)(rows - first), (int)extent, scales ? (const char *)scales + first * (pitch / 16) : nullptr};
  }
};

// What the last workgroups of a product's launch do besides: nothing, or work that was ready before it.
struct NoTail {
  static constexpr bool kAny = false;
  int blocks() const { return 0; }
};

template <class B, int KIND, int BM, int BN, bool ACROSS_A, bool ACROSS_B, bool TWO_B, class Epilogue, class Tail>
__global__ __launch_bounds__(B::kThreads) void k_product(Matrix a, Matrix b, Blocks blocks, Epilogue epilogue, Tail tail) {
  __shared__ __attribute__((aligned(1024))) char lds[B::kLds];
  int r, c, split, total = gridDim.x;
  if constexpr (Tail::kAny) {
    total -= tail.blocks();
    if ((int)blockIdx.x >= total) return tail(blockIdx.x - total, B::kThreads, lds);
  }
  blocks.locate(blockIdx.x, total, r, c, split);
  r = tile::uniform(r);
  c = tile::uniform(c);
  int s0, s1;
  blocks.range(split, s0, s1);
  const int64_t row0 = (int64_t)r * BM + B::row0(), col0 = (int64_t)c * BN + B::col0();
  B block;
  block.run(a.template at<KIND, BM, ACROSS_A>(r), b.template at<KIND, BN, ACROSS_B, TWO_B>(c), s0, s1, lds);
  if (B::holds()) epilogue(block, row0, col0, split, r != c);
}

// Launches the blocks of one shape. What the sizes need of it is the caller's rule.
template <int KIND, int BM, int BN, int WM, int WN, int STAGES, int GROUPS, bool ACROSS_A, bool ACROSS_B, bool TWO_B = false, class Epilogue, class Tail>
sdnn_status launch(const Matrix &a, const Matrix &b, int64_t rows, int64_t cols, int64_t k, int splits, const Epilogue &e, hipStream_t stream, const char *what, bool symmetric,
                   int batch, const Tail &tail) {
  using B = tile::Block<KIND, BM, BN, WM, WN, ACROSS_A, ACROSS_B, STAGES, GROUPS, TWO_B>;
  Blocks blocks;
  blocks.slabs = (int)ceil_div(k, tile::Geometry<KIND>::kPerSlab) * tile::Geometry<KIND>::kSlabs;
  blocks.per = (int)ceil_div(blocks.slabs, splits);
  blocks.splits = splits;
  const int64_t r = ceil_div(rows, BM), c = ceil_div(cols, BN);
  const int64_t n = (symmetric ? c * (c + 1) / 2 : r * c * splits) + tail.blocks();
  blocks.symmetric = symmetric;
  if (n * B::kThreads > 0xffffffffll || a.pitch > kMaxPitch || b.pitch > kMaxPitch || b.pitch_second > kMaxPitch) return fail(SDNN_EINVAL, "%s: %lld x %lld outputs are too many for one launch", what, (long long)rows, (long long)cols);
  blocks.rows = (int)r;
  blocks.cols = (int)c;
  hipLaunchKernelGGL((k_product<B, KIND, BM, BN, ACROSS_A, ACROSS_B, TWO_B, Epilogue, Tail>), dim3((unsigned)n, (unsigned)batch), dim3(B::kThreads), 0, stream, a, b, blocks, e, tail);
  return launched(what);
}

// The shapes of a block: outputs, how many a CU holds, microseconds of bf16 that one takes for a slab when the CU is full
// of them (its share) and when it is alone there (kPaired and the last three have two slabs in work at once).
enum Shape { kWide, kBroad, kMiddle, kSquare, kPaired, kStream, kSmall, kFlat, kTall, kShapes };
struct ShapeCost {
  int bm, bn, held;
  double full, alone;
};
constexpr ShapeCost kCost[kShapes] = {{256, 256, 1, 1.65, 1.65}, {256, 192, 1, 1.35, 1.35}, {192, 192, 1, 1.0, 1.0}, {128, 128, 2, 0.5, 0.65}, {128, 128, 1, 0.55, 0.55},
                                      {64, 64, 4, 0.19, 0.25},   {64, 64, 1, 0.19, 0.19},   {32, 128, 1, 0.19, 0.19}, {128, 32, 1, 0.19, 0.19}};

struct Plan {
  Shape shape;
  int splits;
  double us;  // what the model makes of it
};
enum Form { kAnyForm, kAlong };  // kAlong: both operands are (rows of 192 columns make no whole loads)

// The shape and split that a model of the launch finds fastest: rounds of resident blocks times slabs (1.4 as long for
// three products a slab, 2.3 in fp32), and for a split sum its slabs' traffic (at 4 TB/s) and one launch more.
inline Plan plan(int kind, int64_t rows, int64_t cols, int64_t k, int most_splits, Form form = kAnyForm, int64_t batch = 1, bool symmetric = false) {
  const int64_t slabs = kind == tile::KIND_THREE ? 6 * ceil_div(k, 64) : ceil_div(k, kind == tile::KIND_BF16 ? 64 : kind == tile::KIND_MX ? 256 : 32);
  const double longer = kind == tile::KIND_SPLIT ? 1.4 : kind == tile::KIND_F32 ? 2.3 : 1.0;
  Plan best = {kStream, 1, 1e30};
  for (int s = 0; s < kShapes; ++s) {
    const ShapeCost &c = kCost[s];
    if (kind == tile::KIND_F32 && s < kStream) continue;  // memory bounds it: small blocks, of which a CU holds several
    if ((symmetric && c.bm != c.bn) || ((s == kMiddle || s == kBroad) && form != kAlong)) continue;
    const double across = (double)ceil_div(cols, c.bn), blocks = symmetric ? across * (across + 1) / 2 : (double)ceil_div(rows, c.bm) * across;
    for (int split : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
      if (split > most_splits || (split > 1 && split * 2 > slabs)) break;
      const double n = blocks * split * batch, rounds = std::ceil(n / (kCus * c.held));
      const double held = std::min<double>(c.held, std::ceil(n / kCus));
      // (a round's first loads and last stores overlap with other blocks' work where a CU holds several)
      double t = rounds * (longer * (double)ceil_div(slabs, split) * std::max(c.alone, held * c.full) + 5.0 / std::sqrt(held));
      if (split > 1) t += 5.0 + 2e-6 * rows * cols * split * batch;
      if (t < best.us) best = {(Shape)s, split, t};
    }
  }
  return best;
}

// TWO: b is of two matrices (blocks of 192 columns do not split into wave parts of whole pairs).
template <int KIND, bool AA, bool AB, bool TWO = false, class E, class Tail = NoTail>
sdnn_status run_shape(const Plan &p, const Matrix &a, const Matrix &b, int64_t rows, int64_t cols, int64_t k, const E &e, hipStream_t stream, const char *what, bool symmetric = false, int batch = 1,
                      const Tail &tail = {}) {
  constexpr int kPair = KIND == tile::KIND_MX ? 1 : 2;  // (its scales need LDS too: two blocks a CU instead)
  if constexpr (KIND == tile::KIND_F32) {
    switch (p.shape) {
      case kSmall: return launch<KIND, 64, 64, 2, 2, 4, 2, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
      case kFlat: return launch<KIND, 32, 128, 1, 4, 3, 2, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
      case kTall: return launch<KIND, 128, 32, 4, 1, 3, 2, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
      default: return launch<KIND, 64, 64, 2, 2, 2, 1, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    }
  } else {
  switch (p.shape) {
    case kWide: return launch<KIND, 256, 256, 2, 4, 2, 1, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    case kBroad:
      if constexpr (!AA && !AB && !TWO) return launch<KIND, 256, 192, 2, 4, 2, 1, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    case kMiddle:
      if constexpr (!AA && !AB && !TWO) return launch<KIND, 192, 192, 2, 4, 2, 1, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    case kSquare: return launch<KIND, 128, 128, 2, 2, 2, 1, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    case kPaired: return launch<KIND, 128, 128, 2, 2, 2, 2, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    case kStream: return launch<KIND, 64, 64, 2, 2, 2, 1, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    case kSmall: return launch<KIND, 64, 64, 2, 2, 4, kPair, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    case kFlat: return launch<KIND, 32, 128, 1, 4, 3, kPair, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
    default: return launch<KIND, 128, 32, 4, 1, 3, kPair, AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, symmetric, batch, tail);
  }
  }
}

inline sdnn_status check_matrix(const char *name, const void *p, int64_t ld, int64_t cols, int32_t dtype) {
  if (!p) return fail(SDNN_EINVAL, "%s is null", name);
  if ((uintptr_t)p % dtype_bytes(dtype)) return fail(SDNN_EINVAL, "%s is not aligned to its values", name);
  if (ld < cols || ld > (1ll << 40)) return fail(SDNN_EINVAL, "the row stride of %s, %lld, is outside [%lld, 2^40]", name, (long long)ld, (long long)cols);
  return SDNN_OK;
}

inline sdnn_status check_workspace(const void *p, size_t bytes, size_t need) {
  if (bytes < need) return fail(SDNN_ERANGE, "workspace of %zu bytes, %zu needed", bytes, need);
  if (need && (!p || ((uintptr_t)p & 255))) return fail(SDNN_EINVAL, "workspace is null or not 256-byte aligned");
  return SDNN_OK;
}

}  // namespace dense

#endif  // SDNN_DENSE_H
