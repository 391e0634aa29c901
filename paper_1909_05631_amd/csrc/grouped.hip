// Weights held as 4-bit whole numbers with a scale, and perhaps an offset, for every group of 32, 64 or 128 values of a
// row: w = s (q - 8), or s q + o. The rows x that they are multiplied with stay as they are.
//
//   y = sum over groups of  s sum_k x_k q_k + o sum_k x_k      (o = -8 s where there are no offsets)
//
// Few rows (k_few): every byte of codes goes from memory to registers once and from there to the matrix instructions as
// exact whole numbers; a group's scale meets its fp32 sum, not its weights. A lane loads 32 codes of one output; four
// lane exchanges bring the four lane groups of 16 to the same group of 32; a nibble in a byte is an 8-bit float of 2^-9 times
// its value (up to 7 as a denormal number, from 8 on by its exponent), so that one conversion with the scale 2^9 makes two of
// them the bf16 numbers 0 to 15. x is written once into LDS in the order of the codes, in bf16, fp32 as three bf16 parts
// (exactly), with its sums over groups, which start the groups' products at -8 sum x or are multiplied with the offsets.
// Many rows: the weights are written as values of x's type, and the tile products do the rest.
#include "dense.h"
#include "copies.h"
#include "few.h"
#include "sums.h"

using namespace dense;
using namespace copies;
using namespace sums;
using tile::i32x4;
using tile::KIND_BF16;
using tile::KIND_F32;
using tile::KIND_SPLIT;

namespace {

constexpr int64_t kFewRows = 64;               // rows that go to k_few, 16 at a time
constexpr int64_t kPieceValues = 1 << 28;      // weights that are written as values at a time
constexpr int64_t kPlain = 192;                // fp32 rows or outputs for the plain fp32 products

__host__ __device__ inline int64_t groups_of(int64_t n, int group) { return ceil_div(n, group); }
__host__ __device__ inline int64_t pitch_of(int64_t n, int group) { return groups_of(n, group) * (group / 2); }  // bytes of a row of codes
inline bool good_group(int64_t g) { return g == 32 || g == 64 || g == 128; }

// ------------------------------------------------------------------------------------------------
// Quantisation and its inverse

template <class T>
__device__ __forceinline__ float rounded(float v) { return (float)(T)v; }

// Eight values a lane, GROUP / 8 lanes a group. The scale and offset are rounded to the weights' type before codes are taken
// with them, so that these are the nearest to what they will stand for.
template <class T, int GROUP, bool OFFSETS>
__global__ __launch_bounds__(256) void k_quantize(const T *w, int64_t ld, int64_t rows, int64_t n, bool vec, uint8_t *codes, T *scales, T *offsets) {
  const int64_t groups = groups_of(n, GROUP), per = groups * (GROUP / 8);
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y) {
    const T *row = w + r * ld;
    const int64_t last = ceil_div(per, 64) * 64;  // whole waves: a group's lanes stay together
    for (int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x; c < last; c += (int64_t)gridDim.x * 256) {
      float v[8], low = __builtin_inff(), high = -__builtin_inff();
      bool bad = false;
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const f32x4 x = c < per ? few::load4(row, (int)(c * 8 + i), (int)n, vec) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[i + e] = x[e];
          if (c * 8 + i + e < n) {
            bad |= !__builtin_isfinite(x[e]);
            low = fminf(low, x[e]);
            high = fmaxf(high, x[e]);
          }
        }
      }
#pragma unroll
      for (int d = 1; d < GROUP / 8; d <<= 1) {
        low = fminf(low, __shfl_xor(low, d));
        high = fmaxf(high, __shfl_xor(high, d));
        bad |= __shfl_xor((int)bad, d) != 0;
      }
      const float offset = OFFSETS ? rounded<T>(low) : 0.0f;
      // (a range past the largest number is no infinity this way)
      const float scale = bad ? __builtin_nanf("") : rounded<T>(OFFSETS ? high / 15.0f - low / 15.0f : fmaxf(-low, high) / 7.0f);
      uint32_t word = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float q = OFFSETS ? 0.0f : 8.0f;
        if (c * 8 + i < n && scale > 0.0f) q = OFFSETS ? fminf(fmaxf(rintf((v[i] - offset) / scale), 0.0f), 15.0f) : fminf(fmaxf(rintf(v[i] / scale), -8.0f), 7.0f) + 8.0f;
        word |= (uint32_t)q << 4 * i;
      }
      if (c < per) {
        *(uint32_t *)(codes + r * pitch_of(n, GROUP) + c * 4) = word;
        if (c % (GROUP / 8) == 0) {
          scales[r * groups + c / (GROUP / 8)] = (T)scale;
          if (OFFSETS) offsets[r * groups + c / (GROUP / 8)] = (T)(bad ? __builtin_nanf("") : offset);
        }
      }
    }
  }
}

// Eight values a lane: one product and sum in fp32, rounded to the output's type. Zeros past n, where the output has room.
template <class T>
__global__ __launch_bounds__(256) void k_dequantize(const uint8_t *codes, const T *scales, const T *offsets, int group, int64_t rows, int64_t n, T *out, int64_t ld, int64_t wide, bool vec) {
  const int64_t groups = groups_of(n, group), pitch = pitch_of(n, group);
  for (int64_t r = blockIdx.y; r < rows; r += gridDim.y)
    for (int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; c < wide; c += (int64_t)gridDim.x * 2048) {
      const uint32_t word = c < n ? *(const uint32_t *)(codes + r * pitch + c / 2) : 0;
      const int64_t g = r * groups + (c < n ? c / group : 0);
      const float scale = (float)scales[g], offset = offsets ? (float)offsets[g] : 0.0f, from = offsets ? 0.0f : 8.0f;
      f32x4 v[2];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i / 4][i % 4] = c + i < n ? fmaf((float)(word >> 4 * i & 15) - from, scale, offset) : 0.0f;
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if (c + 4 * h < wide) store4(out + r * ld + c + 4 * h, v[h], (int)min(wide - c - 4 * h, (int64_t)4), vec);
    }
}

// ------------------------------------------------------------------------------------------------
// Few rows

constexpr int kWaves = 8, kThreads = 64 * kWaves, kStep = 128;  // k of a wave's load
constexpr int kStage = 64 * 1024;                              // bytes of LDS: two workgroups a CU

template <class T>
struct Few {
  const T *x;
  int64_t ldx;
  bool vec_x;
  int rows, n;  // of x (all of them), values of a row
  const uint8_t *codes;
  const T *scales, *offsets;
  int64_t outputs;
  T *out;
  int64_t ldo;
  int parts;  // waves that share an output's k
  int chunk;  // k in LDS at a time: whole steps for every one of them
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));

// A 4 x 4 transposition: word r of lane group j becomes word j of lane group r.
__device__ __forceinline__ i32x4 across_groups(i32x4 v) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const u32x2 a = __builtin_amdgcn_permlane16_swap((unsigned)v[0], (unsigned)v[1], false, false), b = __builtin_amdgcn_permlane16_swap((unsigned)v[2], (unsigned)v[3], false, false);
  const u32x2 c = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
  return i32x4{(int)c[0], (int)d[0], (int)c[1], (int)d[1]};
}

// Eight codes as bf16 numbers, in the order 0 2 4 6 1 3 5 7.
__device__ __forceinline__ bf16x8 numbers(int word) {
  const int even = word & 0x0f0f0f0f, odd = word >> 4 & 0x0f0f0f0f;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 512.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(even, 512.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 512.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(odd, 512.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <class T, int GROUP, bool OFFSETS>
__global__ __launch_bounds__(kThreads) void k_few(Few<T> p) {
  constexpr int kParts = sizeof(T) == 4 ? 3 : 1;  // of x
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = tile::uniform(tid >> 6), i16 = lane & 15, j4 = lane >> 4;
  const int t0 = blockIdx.y * 16, rows = min(p.rows - t0, 16);
  const int pitch_x = p.chunk * 2 * kParts + 16;  // 16 bytes on, so that the rows of a fragment lie in different banks
  const int fours = (rows + 3) / 4;
  f32x4 *room = (f32x4 *)lds;                                   // a wave's 16 x 16 sums
  f32x4 *sums = room + kThreads;                                // [group][rows / 4]: sums of x, times -8 without offsets
  char *const stage = (char *)(sums + p.chunk / GROUP * fours);  // x
  const int64_t pitch = pitch_of(p.n, GROUP), groups = groups_of(p.n, GROUP);
  const int part = wave % p.parts, member = wave / p.parts, tiles = kWaves / p.parts;
  const bool once = p.chunk >= p.n;
  const char *frag = stage + min(i16, rows - 1) * pitch_x + j4 * 16;
  const int64_t turns = ceil_div(p.outputs, 16 * tiles);
  for (int64_t turn = blockIdx.x; turn < turns; turn += gridDim.x) {
    const int64_t first = (turn * tiles + member) * 16;
    const int there = (int)max((int64_t)0, min(p.outputs - first, (int64_t)16));
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void *)(p.codes + first * pitch), 0, there * (int)pitch, 0x00027000);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)(p.scales + first * groups), 0, there * (int)groups * (int)sizeof(T), 0x00027000);
    const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc((void *)(p.offsets + first * groups), 0, OFFSETS ? there * (int)groups * (int)sizeof(T) : 0, 0x00027000);
    const auto value = [&](__amdgpu_buffer_rsrc_t r, int g) {  // of group g of this lane's output; zero past the last
      const int at = g < (int)groups ? (i16 * (int)groups + g) * (int)sizeof(T) : (int)tile::kOut;
      if constexpr (sizeof(T) == 4)
        return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, at, 0, 0));
      else
        return (float)__builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(r, at, 0, 0));
    };
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int k0 = 0; k0 < p.n; k0 += p.chunk) {
      if (!once || turn == blockIdx.x) {
        __syncthreads();
        const int units = p.chunk / 8;  // a multiple of 16: a group's lanes stay together
        for (int u = tid; u < rows * units; u += kThreads) {
          const int r = u / units, k = (u - r * units) * 8;
          const T *row = p.x + (t0 + r) * p.ldx;
          const f32x4 a = few::load4(row, k0 + k, p.n, p.vec_x), b = few::load4(row, k0 + k + 4, p.n, p.vec_x);
          const float v[8] = {a[0], a[2], b[0], b[2], a[1], a[3], b[1], b[3]};
          bf16x8 out[kParts];
          float sum = 0.0f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            sum += v[i];
            if constexpr (kParts == 3) {
              __bf16 h, m, l;
              split3(v[i], h, m, l);
              out[0][i] = h;
              out[1][i] = m;
              out[2][i] = l;
            } else {
              out[0][i] = (__bf16)v[i];
            }
          }
          char *to = stage + r * pitch_x + k / 32 * (64 * kParts) + k % 32 * 2;
#pragma unroll
          for (int i = 0; i < kParts; ++i) *(bf16x8 *)(to + 64 * i) = out[i];
#pragma unroll
          for (int d = 1; d < GROUP / 8; d <<= 1) sum += __shfl_xor(sum, d);
          if (k % GROUP == 0) ((float *)sums)[k / GROUP * 4 * fours + r] = OFFSETS ? sum : -8.0f * sum;
        }
        __syncthreads();
      }
      const int steps = min(p.chunk, (int)ceil_div(p.n - k0, kStep) * kStep) / kStep;
      const int per = (steps + p.parts - 1) / p.parts, s1 = min((part + 1) * per, steps);
      constexpr int U = 4, G = kStep / GROUP;
      for (int s = part * per; s < s1; s += U) {
        i32x4 c[U];
        float scale[U][G], offset[U][G];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int at = (k0 + (s + u) * kStep) / 2 + j4 * 16;
          c[u] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, s + u < s1 && at < (int)pitch ? i16 * (int)pitch + at : (int)tile::kOut, 0, 0));
#pragma unroll
          for (int g = 0; g < G; ++g) {
            const int which = s + u < s1 ? (k0 + (s + u) * kStep) / GROUP + g : (int)groups;
            scale[u][g] = value(rs, which);
            if constexpr (OFFSETS) offset[u][g] = value(ro, which);
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int step = min(s + u, s1 - 1);  // past the last: codes, scales and offsets of zero
          const i32x4 words = across_groups(c[u]);
          f32x4 sum;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int g = q * 32 / GROUP;
            if (q * 32 % GROUP == 0) {
              const f32x4 x = sums[(step * G + g) * fours + min(j4, fours - 1)];  // (past the rows: anything)
              if constexpr (OFFSETS) {
                sum = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = fmaf(offset[u][g], x[e], acc[e]);
              } else {
                sum = x;
              }
            }
            const bf16x8 w = numbers(words[q]);
            const char *a = frag + (step * 4 + q) * (64 * kParts);
#pragma unroll
            for (int i = kParts - 1; i >= 0; --i) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8 *)(a + 64 * i), w, sum, 0, 0, 0);
            if ((q + 1) * 32 % GROUP == 0)
#pragma unroll
              for (int e = 0; e < 4; ++e) acc[e] = fmaf(scale[u][g], sum[e], acc[e]);
          }
        }
      }
    }
    if (p.parts > 1) {
      __syncthreads();
      room[wave * 64 + lane] = acc;
      __syncthreads();
      if (part == 0)
        for (int i = 1; i < p.parts; ++i) acc += room[(wave + i) * 64 + lane];
    }
    if (part == 0 && i16 < there)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (4 * j4 + e < rows) p.out[(t0 + 4 * j4 + e) * p.ldo + first + i16] = (T)acc[e];
  }
}

template <class T, int GROUP>
sdnn_status few_of(Few<T> p, hipStream_t stream) {
  const int parts_x = sizeof(T) == 4 ? 3 : 1, rows = std::min(p.rows, 16);
  const int64_t tiles = ceil_div(p.outputs, 16), steps = ceil_div(p.n, kStep);
  const int64_t fours = ceil_div(rows, 4) * 16, per_step = rows * kStep * 2 * parts_x + kStep / GROUP * fours, fixed = kThreads * 16 + rows * 16;
  const int64_t fit = (kStage - fixed) / per_step;  // steps of k: 4 at least (16 rows in three parts, groups of 32)
  // as many waves on one output's k as it takes to give every CU two workgroups
  p.parts = 1;
  while (p.parts < kWaves && tiles * p.parts < kWaves * 2 * kCus && p.parts * 2 <= std::min(steps, fit)) p.parts *= 2;
  const int64_t unit = kStep * p.parts;
  p.chunk = (int)std::min(fit / p.parts * unit, ceil_div(p.n, unit) * unit);
  const size_t lds = (size_t)(fixed + p.chunk / kStep * per_step);
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(tiles * p.parts, kWaves), 2 * kCus), (unsigned)ceil_div(p.rows, 16));
  if (p.offsets)
    hipLaunchKernelGGL((k_few<T, GROUP, true>), grid, dim3(kThreads), lds, stream, p);
  else
    hipLaunchKernelGGL((k_few<T, GROUP, false>), grid, dim3(kThreads), lds, stream, p);
  return launched("linear");
}

// ------------------------------------------------------------------------------------------------
// Many rows

// Sums of two-part operands, whose rows' exponents are taken back, stored in fp32.
struct StoreScaled {
  const int *ex, *ew;
  float *out;
  int64_t ld, rows, cols;
  bool vec;
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
    const int i16 = threadIdx.x & 15, j4 = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t t = row0 + 16 * i + i16;
      const bool in = t < rows;
      const int e = in ? ex[t] : 0;
      store_row<float, B::kTN>(out + t * ld, col0, cols, vec, in, [&](int j) {
        f32x4 v = block.acc[i][j];
        const int64_t c = col0 + 16 * j + 4 * j4;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = ldexpf(v[k], -e - (c + k < cols ? ew[c + k] : 0));
        return v;
      });
    }
  }
};

struct Sizes {
  int64_t rows, outputs, n;
  int32_t dtype;
  bool few() const { return rows <= kFewRows; }
  int kind() const { return dtype == SDNN_BF16 ? KIND_BF16 : std::min(rows, outputs) <= kPlain ? KIND_F32 : KIND_SPLIT; }
  int64_t values() const { return ceil_div(n, 8) * 8; }  // of a row of weights written as values
  int64_t piece() const { return std::min(outputs, std::max<int64_t>(256, kPieceValues / values() / 256 * 256)); }
  int64_t pitch() const { return kind() == KIND_SPLIT ? ceil_div(n, 32) * 128 : values() * dtype_bytes(dtype); }  // of a row of x
};

struct Space {
  char *w, *x, *split;
  int *ex, *ew;
  Space(Carver &c, const Sizes &s) {
    const bool parts = !s.few() && s.kind() == KIND_SPLIT;
    w = c.take<char>(s.few() ? 0 : (size_t)(s.piece() * s.values() * dtype_bytes(s.dtype)));
    x = c.take<char>(s.few() ? 0 : (size_t)(s.rows * s.pitch()));
    split = c.take<char>(parts ? (size_t)(s.piece() * s.pitch()) : 0);
    ex = c.take<int>(parts ? s.rows : 0);
    ew = c.take<int>(parts ? s.piece() : 0);
  }
};

// Workgroups along a row of `items` lanes, and down the rows.
dim3 grid_of(int64_t rows, int64_t items) {
  const int64_t x = ceil_div(items, 256);
  return dim3((unsigned)x, (unsigned)std::max<int64_t>(1, std::min<int64_t>({rows, 65535, ceil_div(kCus * 32, x)})));
}

template <class T>
sdnn_status dequantize(const uint8_t *codes, const T *scales, const T *offsets, int group, int64_t rows, int64_t n, T *out, int64_t ld, int64_t wide, hipStream_t stream) {
  hipLaunchKernelGGL((k_dequantize<T>), grid_of(rows, ceil_div(wide, 8)), dim3(256), 0, stream, codes, scales, offsets, group, rows, n, out, ld, wide, vector_rows(out, ld));
  return launched("dequantize");
}

template <int KIND, class T>
sdnn_status many(const Sizes &s, const T *x, int64_t ldx, const uint8_t *codes, const T *scales, const T *offsets, int group, T *out, int64_t ldo, const Space &sp, hipStream_t stream) {
  Sources src{};
  src.cols = s.n;
  src.of[0] = {x, ldx, s.rows, sp.x, sp.ex, aligned16(x, ldx, sizeof(T))};
  Matrix a{sp.x, s.pitch(), s.rows, s.pitch(), 0};
  const dim3 grid((unsigned)std::min<int64_t>(s.rows, 4096));
  if constexpr (KIND == KIND_SPLIT)
    hipLaunchKernelGGL(k_two_parts, grid, dim3(256), 0, stream, src, s.rows);
  else if (usable_in_place(x, ldx, s.n, sizeof(T)))
    a = {(const char *)x, ldx * (int64_t)sizeof(T), s.rows, s.n * (int64_t)sizeof(T), 0};
  else
    hipLaunchKernelGGL((k_aligned<T>), grid, dim3(256), 0, stream, src, s.rows);
  sdnn_status st = launched("linear");
  const int64_t groups = groups_of(s.n, group), piece = s.piece(), ld = s.values();
  for (int64_t v0 = 0; v0 < s.outputs && st == SDNN_OK; v0 += piece) {
    const int64_t m = std::min(piece, s.outputs - v0);
    st = dequantize(codes + v0 * pitch_of(s.n, group), scales + v0 * groups, offsets ? offsets + v0 * groups : nullptr, group, m, s.n, (T *)sp.w, ld, ld, stream);
    if (st != SDNN_OK) return st;
    Matrix b{sp.w, ld * (int64_t)sizeof(T), m, a.extent, 0};
    if constexpr (KIND == KIND_SPLIT) {
      Sources w{};
      w.cols = s.n;
      w.of[0] = {sp.w, ld, m, sp.split, sp.ew, true};
      hipLaunchKernelGGL(k_two_parts, dim3((unsigned)std::min<int64_t>(m, 4096)), dim3(256), 0, stream, w, m);
      if ((st = launched("linear")) != SDNN_OK) return st;
      b = {sp.split, s.pitch(), m, s.pitch(), 0};
      const StoreScaled e{sp.ex, sp.ew, out + v0, ldo, s.rows, m, vector_rows(out + v0, ldo)};
      st = run_shape<KIND, false, false>(plan(KIND, s.rows, m, s.n, 1, kAlong), a, b, s.rows, m, s.n, e, stream, "linear");
    } else {
      const Store<T> e{out + v0, ldo, s.rows, m, vector_rows(out + v0, ldo)};
      st = run_shape<KIND, false, false>(plan(KIND, s.rows, m, s.n, 1, kAlong), a, b, s.rows, m, s.n, e, stream, "linear");
    }
  }
  return st;
}

template <class T>
sdnn_status linear(const Sizes &s, const void *x, int64_t ldx, const uint8_t *codes, const void *scales, const void *offsets, int group, void *out, int64_t ldo, void *workspace, hipStream_t stream) {
  if (s.few()) {
    const Few<T> p{(const T *)x, ldx, aligned16(x, ldx, sizeof(T)), (int)s.rows, (int)s.n, codes, (const T *)scales, (const T *)offsets, s.outputs, (T *)out, ldo, 0, 0};
    return group == 32 ? few_of<T, 32>(p, stream) : group == 64 ? few_of<T, 64>(p, stream) : few_of<T, 128>(p, stream);
  }
  Carver c{(char *)workspace};
  const Space sp(c, s);
  const auto call = [&](auto kind) { return many<kind(), T>(s, (const T *)x, ldx, codes, (const T *)scales, (const T *)offsets, group, (T *)out, ldo, sp, stream); };
  if constexpr (sizeof(T) == 2)
    return call(std::integral_constant<int, KIND_BF16>{});
  else
    return s.kind() == KIND_F32 ? call(std::integral_constant<int, KIND_F32>{}) : call(std::integral_constant<int, KIND_SPLIT>{});
}

template <class T>
sdnn_status quantize(const T *w, int64_t ld, int64_t rows, int64_t n, int group, uint8_t *codes, T *scales, T *offsets, hipStream_t stream) {
  const dim3 grid = grid_of(rows, groups_of(n, group) * (group / 8));
  const bool vec = vector_rows(w, ld);
  const auto go = [&](auto g) {
    if (offsets)
      hipLaunchKernelGGL((k_quantize<T, g(), true>), grid, dim3(256), 0, stream, w, ld, rows, n, vec, codes, scales, offsets);
    else
      hipLaunchKernelGGL((k_quantize<T, g(), false>), grid, dim3(256), 0, stream, w, ld, rows, n, vec, codes, scales, offsets);
  };
  if (group == 32)
    go(std::integral_constant<int, 32>{});
  else if (group == 64)
    go(std::integral_constant<int, 64>{});
  else
    go(std::integral_constant<int, 128>{});
  return launched("quantize");
}

sdnn_status check_shape(int64_t n_rows, int64_t n_values, int32_t group, int32_t dtype) {
  if (n_rows < 0 || n_rows > kMaxRows) return fail(SDNN_EINVAL, "n_rows %lld is outside [0, %lld]", (long long)n_rows, (long long)kMaxRows);
  if (n_values < 1 || n_values > kMaxFeatures) return fail(SDNN_EINVAL, "n_values %lld is outside [1, %lld]", (long long)n_values, (long long)kMaxFeatures);
  if (!good_group(group)) return fail(SDNN_EINVAL, "group %d is none of 32, 64 and 128", group);
  if (!good_dtype(dtype)) return fail(SDNN_EINVAL, "dtype %d is neither SDNN_FP32 nor SDNN_BF16", dtype);
  return SDNN_OK;
}

sdnn_status check_codes(const uint8_t *codes, const void *scales, const void *offsets, int32_t dtype) {
  if (!codes || !scales) return fail(SDNN_EINVAL, "codes or scales are null");
  if ((uintptr_t)codes & 15) return fail(SDNN_EINVAL, "codes are not 16-byte aligned");
  if ((uintptr_t)scales % dtype_bytes(dtype) || (uintptr_t)offsets % dtype_bytes(dtype)) return fail(SDNN_EINVAL, "scales or offsets are not aligned to their values");
  return SDNN_OK;
}

}  // namespace

extern "C" {

int64_t sdnn_grouped_groups(int64_t n_values, int32_t group) { return n_values < 1 || n_values > kMaxFeatures || !good_group(group) ? 0 : groups_of(n_values, group); }

sdnn_status sdnn_grouped_quantize(const void *w, int64_t ldw, int32_t dtype, int64_t n_rows, int64_t n_values, int32_t group, uint8_t *codes, void *scales, void *offsets, void *hip_stream) {
  sdnn_status st = check_shape(n_rows, n_values, group, dtype);
  if (st != SDNN_OK || n_rows == 0) return st;
  if ((st = check_matrix("w", w, ldw, n_values, dtype)) != SDNN_OK) return st;
  if ((st = check_codes(codes, scales, offsets, dtype)) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  return dtype == SDNN_BF16 ? quantize((const __bf16 *)w, ldw, n_rows, n_values, group, codes, (__bf16 *)scales, (__bf16 *)offsets, stream)
                            : quantize((const float *)w, ldw, n_rows, n_values, group, codes, (float *)scales, (float *)offsets, stream);
}

sdnn_status sdnn_grouped_dequantize(const uint8_t *codes, const void *scales, const void *offsets, int32_t dtype, int64_t n_rows, int64_t n_values, int32_t group, void *out, int64_t ldo,
                                    void *hip_stream) {
  sdnn_status st = check_shape(n_rows, n_values, group, dtype);
  if (st != SDNN_OK || n_rows == 0) return st;
  if ((st = check_codes(codes, scales, offsets, dtype)) != SDNN_OK) return st;
  if ((st = check_matrix("out", out, ldo, n_values, dtype)) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  return dtype == SDNN_BF16 ? dequantize(codes, (const __bf16 *)scales, (const __bf16 *)offsets, group, n_rows, n_values, (__bf16 *)out, ldo, n_values, stream)
                            : dequantize(codes, (const float *)scales, (const float *)offsets, group, n_rows, n_values, (float *)out, ldo, n_values, stream);
}

size_t sdnn_grouped_linear_workspace_bytes(int64_t n_rows, int64_t n_outputs, int64_t n_values, int32_t dtype) {
  if (check_shape(n_rows, n_values, 32, dtype) != SDNN_OK || n_outputs < 0 || n_outputs > kMaxClasses || n_rows == 0 || n_outputs == 0) return 0;
  Carver c{nullptr};
  Space sp(c, {n_rows, n_outputs, n_values, dtype});
  return c.used;
}

sdnn_status sdnn_grouped_linear(const void *x, int64_t ldx, int32_t dtype, const uint8_t *codes, const void *scales, const void *offsets, int64_t n_rows, int64_t n_outputs, int64_t n_values,
                                int32_t group, void *out, int64_t ldo, void *workspace, size_t workspace_bytes, void *hip_stream) {
  sdnn_status st = check_shape(n_rows, n_values, group, dtype);
  if (st != SDNN_OK) return st;
  if (n_outputs < 0 || n_outputs > kMaxClasses) return fail(SDNN_EINVAL, "n_outputs %lld is outside [0, %lld]", (long long)n_outputs, (long long)kMaxClasses);
  if (n_rows == 0 || n_outputs == 0) return SDNN_OK;
  if ((st = check_matrix("x", x, ldx, n_values, dtype)) != SDNN_OK) return st;
  if ((st = check_codes(codes, scales, offsets, dtype)) != SDNN_OK) return st;
  if ((st = check_matrix("out", out, ldo, n_outputs, dtype)) != SDNN_OK) return st;
  if ((st = check_workspace(workspace, workspace_bytes, sdnn_grouped_linear_workspace_bytes(n_rows, n_outputs, n_values, dtype))) != SDNN_OK) return st;
  const Sizes s{n_rows, n_outputs, n_values, dtype};
  const hipStream_t stream = (hipStream_t)hip_stream;
  return dtype == SDNN_BF16 ? linear<__bf16>(s, x, ldx, codes, scales, offsets, group, out, ldo, workspace, stream)
                            : linear<float>(s, x, ldx, codes, scales, offsets, group, out, ldo, workspace, stream);
}

}  // extern "C"
