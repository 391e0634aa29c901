// Weights held as 4-bit whole numbers with a scale, and perhaps an offset, for every group of 32, 64 or 128 values of a
// row: w = s (q - 8), or s q + o. The rows x that they are multiplied with stay as they are.
//
//   y = sum over groups of  s sum_k x_k q_k + o sum_k x_k      (o = -8 s where there are no offsets)
//
// Few rows (k_few): every byte of codes goes from memory to registers once and from there to the matrix instructions as
// exact whole numbers; a group's scale meets its fp32 sum, not its weights. A lane loads 32 codes of one output, so that 16
// lanes of each of 4 groups read 64 bytes of a row; four lane exchanges bring the four lane groups to the same 32 codes' group.
// A nibble in a byte is an 8-bit float of 2^-9 times its value (up to 7 as a denormal number, from 8 on by its exponent), so
// that one conversion with the scale 2^9 makes two of them the bf16 numbers 0 to 15. x stays in a workgroup's LDS, in bf16,
// fp32 as three bf16 parts (exactly), past its size in slices of k whose sums a second kernel joins. Its sums over groups
// are one more product, with a row of ones, or of -8.
// Bound by the codes' bytes for one row (1 x 4096 to 65536 outputs 28.6 us, 4.8 TB/s; 1 x 16384 to 16384 30 us). Each 16 rows
// more are one more product, LDS read and sum for each of them, and x takes its time on the way to LDS: 16 x 16384 to 16384
// 38 us, with groups of 64 and offsets 42; 64 rows 75.
// Many rows: the weights are written as values of x's type, rounded to it, and the tile products do the rest (2000 x 4096 to
// 16384 outputs 253 us, 30 of them for that).
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

constexpr int64_t kFewRows = 64;               // rows that k_few takes at once
constexpr int64_t kManyWeights = 1 << 24, kManyOutputs = 4096;  // see Sizes::few
// Weights that are written as values at a time. Fewer (2^26 bf16 values would stay in the Infinity Cache) leave the products too
// few blocks: 512 x 16384 to 16384 478 us so, 388 at once; 2000 rows 1037 and 960.
constexpr int64_t kPieceValues = 1 << 28;
constexpr int64_t kSplitResults = 1 << 24;  // results of a product whose k may be split: past that there is a 256 x 256 block for every CU
// fp32 rows or outputs (the fewer of the two) for the plain fp32 products. us, plain and in two fp16 parts: 192 x 1000 to 2048 27 / 32,
// 1000 x 1000 to 192 19 / 26, 300 x 1000 to 2048 33 / 33, 300 x 4096 to 8192 229 / 210, 600 x 600 to 600 22 / 22.
constexpr int64_t kPlain = 192;

__host__ __device__ inline int64_t groups_of(int64_t n, int group) { return ceil_div(n, group); }
__host__ __device__ inline int64_t pitch_of(int64_t n, int group) { return groups_of(n, group) * (group / 2); }  // bytes of a row of codes
inline bool good_group(int64_t g) { return g == 32 || g == 64 || g == 128; }

// ------------------------------------------------------------------------------------------------
// Quantisation and its inverse

template <class T>
__device__ __forceinline__ float rounded(float v) { return (float)(T)v; }

// (high - low) / 15. Within a factor of two of each other (of one sign) their difference is exact, and quotients of each could
// cancel to nothing of it (low 1, high the next number). Others lose at most two bits as quotients, whose difference passes no largest
// number.
__device__ __forceinline__ float step_of(float low, float high) {
  const float range = high - low;
  const bool near = range <= 0.5f * fmaxf(-low, high);
  const float step = high / 15.0f - low / 15.0f;
  return __builtin_expect(near, false) ? range / 15.0f : step;
}

// The next number below a scale whose largest code's value would be rounded to infinity.
template <class T>
__device__ __forceinline__ float finite_scale(float scale, float codes, float offset) {
  return rounded<T>(fmaf(codes, scale, offset)) == __builtin_inff() ? __uint_as_float(__float_as_uint(scale) - (sizeof(T) == 2 ? 0x10000u : 1u)) : scale;
}

// Eight values a lane, GROUP / 8 lanes a group. The scale and offset are rounded to the weights' type before codes are taken
// with them, so that these are the nearest to what they will stand for. 16384 x 4096 in groups of 128: bf16 58 us, 63 with offsets
// (168 MB, 34 us at a copy's rate; instructions bound it, a few more for each group cost 4%), fp32 69 and 73 (302 MB, 62 us).
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
      float scale = bad ? __builtin_nanf("") : rounded<T>(OFFSETS ? step_of(low, high) : fmaxf(-low, high) / 7.0f), from = offset, by = scale;
      if (__builtin_expect(fmaxf(-low, high) > 0x1p127f, false)) {  // the rest go past this: 57.9 us (bf16, no offsets) and not 60.7
        by = scale = finite_scale<T>(scale, OFFSETS ? 15.0f : 7.0f, offset);
        if (OFFSETS && !__builtin_isfinite(high - low)) {  // halves' differences are finite, and exact halves: the scale is 2^124 or more
#pragma unroll
          for (int i = 0; i < 8; ++i) v[i] *= 0.5f;
          from *= 0.5f;
          by *= 0.5f;
        }
      }
      uint32_t word = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float q = OFFSETS ? 0.0f : 8.0f;
        if (c * 8 + i < n && scale > 0.0f) q = OFFSETS ? fminf(fmaxf(rintf((v[i] - from) / by), 0.0f), 15.0f) : fminf(fmaxf(rintf(v[i] / by), -8.0f), 7.0f) + 8.0f;
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

// Eight values a lane of four rows: one product and sum in fp32, rounded to the output's type. Zeros past n, where the output
// has room. `shift`: a group is 2^shift values.
template <class T>
__global__ __launch_bounds__(256) void k_dequantize(const uint8_t *codes, const T *scales, const T *offsets, int shift, int64_t rows, int n, T *out, int64_t ld, int wide, bool vec) {
  constexpr int kRows = 4;  // whose loads are on their way together
  const int64_t groups = groups_of(n, 1 << shift), pitch = pitch_of(n, 1 << shift);
  const float from = offsets ? 0.0f : 8.0f;
  for (int64_t r0 = (int64_t)blockIdx.y * kRows; r0 < rows; r0 += (int64_t)gridDim.y * kRows)
    for (int c = (blockIdx.x * 256 + threadIdx.x) * 8; c < wide; c += gridDim.x * 2048) {
      const int at = c < n ? c : 0;
      uint32_t word[kRows];
      float scale[kRows], offset[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int64_t r = min(r0 + i, rows - 1), g = r * groups + (at >> shift);
        word[i] = *(const uint32_t *)(codes + r * pitch + at / 2);
        scale[i] = (float)scales[g];
        offset[i] = offsets ? (float)offsets[g] : 0.0f;
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        if (r0 + i >= rows) break;
        f32x4 v[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e / 4][e % 4] = c + e < n ? fmaf((float)(word[i] >> 4 * e & 15) - from, scale[i], offset[i]) : 0.0f;
        T *to = out + (r0 + i) * ld + c;
        typedef T Eight __attribute__((ext_vector_type(8)));
        if (vec && c + 8 <= wide) {
          Eight o;
#pragma unroll
          for (int e = 0; e < 8; ++e) o[e] = (T)v[e / 4][e % 4];
          *(Eight *)to = o;
        } else {
#pragma unroll
          for (int h = 0; h < 2; ++h)
            if (c + 4 * h < wide) store4(to + 4 * h, v[h], min(wide - c - 4 * h, 4), vec);
        }
      }
    }
}

// ------------------------------------------------------------------------------------------------
// Few rows

constexpr int kStep = 128;  // k of a wave's load

// Parts of a value of x as the matrix instructions take it: bf16, or, fp32, three of them.
template <class T>
constexpr int kPartsOf = sizeof(T) == 4 ? 3 : 1;

template <class T>
struct Few {
  const T *x;
  int64_t ldx;
  bool vec_x;
  int rows, n;
  const uint8_t *codes;
  const T *scales, *offsets;
  int groups, pitch;  // of a row of codes: groups, bytes
  int64_t outputs;
  T *out;
  int64_t ldo;
  float *slabs;  // sums of the slices of k, [slice][row][ld_slab]; nullptr: one slice, stored in out
  int64_t ld_slab;
  int slice;  // steps of a slice
  bool pairs;  // rows of scales and offsets are whole dwords
  int parts;  // waves that share an output's k
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));

// A 4 x 4 transposition: word r of lane group j becomes word j of lane group r.
__device__ __forceinline__ i32x4 across_groups(i32x4 v) {
  const u32x2 a = __builtin_amdgcn_permlane16_swap((unsigned)v[0], (unsigned)v[1], false, false), b = __builtin_amdgcn_permlane16_swap((unsigned)v[2], (unsigned)v[3], false, false);
  const u32x2 c = __builtin_amdgcn_permlane32_swap(a[0], b[0], false, false), d = __builtin_amdgcn_permlane32_swap(a[1], b[1], false, false);
  return i32x4{(int)c[0], (int)d[0], (int)c[1], (int)d[1]};
}

// Eight codes as bf16 numbers.
__device__ __forceinline__ bf16x8 numbers(int word) {
  const unsigned even = word & 0x0f0f0f0f, odd = word >> 4 & 0x0f0f0f0f;
  const unsigned low = __builtin_amdgcn_perm(odd, even, 0x05010400), high = __builtin_amdgcn_perm(odd, even, 0x07030602);  // bytes in their order
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 512.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(low, 512.0f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 512.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(high, 512.0f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// x in LDS: for every row, blocks of 32 values, 64 bytes for each part; rows are 16 bytes more apart, so that those of a
// fragment lie in different banks.
template <class T>
__host__ __device__ inline int stage_pitch(int steps) { return steps * (kStep * 2 * kPartsOf<T>) + 16; }

// Eight values at value `at` of a staged row.
template <class T>
__device__ __forceinline__ void store_eight(char *row, int at, const f32x4 (&v)[2]) {
  constexpr int kParts = kPartsOf<T>;
  bf16x8 out[kParts];
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if constexpr (kParts == 3) {
      __bf16 hi, mid, lo;
      split3(v[i / 4][i % 4], hi, mid, lo);
      out[0][i] = hi;
      out[1][i] = mid;
      out[2][i] = lo;
    } else {
      out[0][i] = (__bf16)v[i / 4][i % 4];
    }
  char *to = row + at / 32 * (64 * kParts) + at % 32 * 2;
#pragma unroll
  for (int i = 0; i < kParts; ++i) *(bf16x8 *)(to + 64 * i) = out[i];
}

// Values [k0, k0 + 8 units) of every row, zeros past n. Rows of whole 16 bytes are loaded without branches, four eights a
// lane at once: one at a time their latency is what this takes (64 x 1000 to 1000 outputs: 20 us so).
template <class T>
__device__ __forceinline__ void stage_rows(char *stage, int pitch, const T *x, int64_t ldx, int rows, int n, int k0, int units, bool vec, int threads) {
  const int total = rows * units;
  if (vec && n % 8 == 0) {
    typedef T Eight __attribute__((ext_vector_type(8)));
    for (int u0 = threadIdx.x; u0 < total; u0 += 4 * threads) {
      Eight v[4];
      int r[4], k[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int u = min(u0 + i * threads, total - 1);
        r[i] = u / units;
        k[i] = (u - r[i] * units) * 8;
        v[i] = *(const Eight *)(x + r[i] * ldx + min(k0 + k[i], n - 8));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f32x4 f[2];
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e / 4][e % 4] = k0 + k[i] < n ? (float)v[i][e] : 0.0f;
        store_eight<T>(stage + r[i] * pitch, k[i], f);
      }
    }
  } else {
    for (int u = threadIdx.x; u < total; u += threads) {
      const int r = u / units, k = (u - r * units) * 8;
      const T *row = x + r * ldx;
      const f32x4 f[2] = {few::load4(row, k0 + k, n, vec), few::load4(row, k0 + k + 4, n, vec)};
      store_eight<T>(stage + r * pitch, k, f);
    }
  }
}

// Scales and offsets of 16 groups of 16 outputs, a wave's in LDS (a row's are 4 values apart, which spreads the rows over the
// banks). Memory is read 4 groups a lane at once: their rows are far apart, and a lane's value at a time would fetch
// each of their lines again and again (16 x 16384 to 16384 outputs, groups of 64 with offsets: 59 us so).
constexpr int kHeld = 16, kHeldPitch = kHeld + 4;
template <class T>
struct Four {
  T v[4];
};

// Orders a wave's LDS stores and the reads of what other lanes of it stored. (They are carried out in the order in which the
// wave issues them; this keeps the compiler to it, and costs nothing.)
__device__ __forceinline__ void wave_meets() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Shapes of a workgroup: 16 rows of x in half a CU's LDS or all of it, 32 or 64 rows, whose fragments serve two tiles of
// outputs each. A wave multiplies STEPS steps at a time, with those of the next AHEAD times on their way.
template <int TILES, int OUTS, int STEPS, int AHEAD, int WAVES, int PER_SIMD, int ROOM>
struct Shape {
  static constexpr int kTiles = TILES, kOuts = OUTS, kSteps = STEPS, kAhead = AHEAD, kWaves = WAVES, kPerSimd = PER_SIMD;
  template <class T>
  static constexpr int kHeldBytes = OUTS * 2 * 16 * kHeldPitch * (int)sizeof(T);  // of a wave
  template <class T>
  static constexpr int kStage = (ROOM << 10) - WAVES * kHeldBytes<T>;  // what is left for x
};
using Half = Shape<1, 1, 2, 1, 8, 4, 76>;
using Whole = Shape<1, 1, 2, 1, 16, 4, 158>;
using Two = Shape<2, 2, 1, 1, 8, 2, 158>;
using FourTiles = Shape<4, 2, 1, 1, 8, 2, 158>;

// TILES x 16 rows (those past the last repeat it; their sums go nowhere), OUTS x 16 outputs a wave at a time. A workgroup
// holds its slice of x in LDS and goes over the outputs; waves in teams of `parts` share an output's k.
template <class T, int SHIFT, bool OFFSETS, class S>
__global__ __launch_bounds__(64 * S::kWaves, S::kPerSimd) void k_few(Few<T> p) {
  constexpr int TILES = S::kTiles, OUTS = S::kOuts, STEPS = S::kSteps, AHEAD = S::kAhead, WAVES = S::kWaves;
  constexpr int kParts = kPartsOf<T>, kGroups = 4 >> SHIFT;  // kGroups: of a step
  // -8 sum x starts each block of 32's sum, so that these never grow far past their result. bf16 rows that serve several
  // tiles of outputs have it for a whole group at once, in one chain for all of them: 3 bits of fp32 less, none of bf16's.
  constexpr bool kWhole = !OFFSETS && OUTS > 1 && kParts == 1;
  __shared__ __attribute__((aligned(16))) char stage[S::template kStage<T>];
  __shared__ __attribute__((aligned(16))) char wave_room[WAVES][S::template kHeldBytes<T>];
  static_assert(S::template kHeldBytes<T> >= 1024, "a wave's sums have room there too");
  const int lane = threadIdx.x & 63, wave = tile::uniform(threadIdx.x >> 6), i16 = lane & 15, j4 = lane >> 4;
  const int part = wave % p.parts, member = wave / p.parts, teams = WAVES / p.parts;
  const int blocks = (p.n + 31) / 32, first_step = blockIdx.y * p.slice, steps = min(p.slice, (p.n + kStep - 1) / kStep - first_step);
  const int per = (steps + p.parts - 1) / p.parts, s0 = part * per, s1 = min(s0 + per, steps);
  const int pitch_x = stage_pitch<T>(steps), units = steps * (kStep / 8);
  stage_rows(stage, pitch_x, p.x, p.ldx, p.rows, p.n, first_step * kStep, units, p.vec_x, 64 * WAVES);
  __syncthreads();
  const char *from[TILES];
#pragma unroll
  for (int r = 0; r < TILES; ++r) from[r] = stage + min(r * 16 + i16, p.rows - 1) * pitch_x + j4 * 16;
  T *const held = (T *)wave_room[wave];
  bf16x8 ones;  // for the sums of x: times -8 where there are no offsets
#pragma unroll
  for (int i = 0; i < 8; ++i) ones[i] = (__bf16)(OFFSETS ? 1.0f : -8.0f);
  const int64_t turns = ceil_div(p.outputs, 16 * OUTS * teams);
  for (int64_t turn = blockIdx.x; turn < turns; turn += gridDim.x) {
    const int64_t first = (turn * teams + member) * (16 * OUTS);
    const int there = (int)max((int64_t)0, min(p.outputs - first, (int64_t)(16 * OUTS)));
    const __amdgpu_buffer_rsrc_t rc = __builtin_amdgcn_make_buffer_rsrc((void *)(p.codes + first * p.pitch), 0, there * p.pitch, 0x00027000);
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)(p.scales + first * p.groups), 0, there * p.groups * (int)sizeof(T), 0x00027000);
    const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc((void *)(p.offsets + first * p.groups), 0, OFFSETS ? there * p.groups * (int)sizeof(T) : 0, 0x00027000);
    // This lane's 4 groups of the 16 from g on; zeros past the last.
    const auto load_four = [&](__amdgpu_buffer_rsrc_t r, int o, int g) {
      Four<T> to;
      g += 4 * j4;
      const int at = g < p.groups ? ((o * 16 + i16) * p.groups + g) * (int)sizeof(T) : (int)tile::kOut;
      if constexpr (sizeof(T) == 4) {
        to = __builtin_bit_cast(Four<T>, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
      } else if (p.pairs) {
        to = __builtin_bit_cast(Four<T>, __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) to.v[i] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(r, at + 2 * i, 0, 0));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) to.v[i] = g + i < p.groups ? to.v[i] : (T)0.0f;
      return to;
    };
    struct Codes {
      i32x4 of[STEPS][OUTS];
    };
    // Of the steps from s on; past s1 and past the last block, zeros.
    const auto load = [&](Codes &to, int s) {
#pragma unroll
      for (int u = 0; u < STEPS; ++u) {
        const int block = (first_step + s + u) * 4 + j4;
#pragma unroll
        for (int o = 0; o < OUTS; ++o)
          to.of[u][o] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rc, s + u < s1 && block < blocks ? (o * 16 + i16) * p.pitch + block * 16 : (int)tile::kOut, 0, 0));
      }
    };
    f32x4 acc[TILES][OUTS];
#pragma unroll
    for (int r = 0; r < TILES; ++r)
#pragma unroll
      for (int o = 0; o < OUTS; ++o) acc[r][o] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    Four<T> next_scales[OUTS], next_offsets[OUTS];
    int next = (first_step + s0) * 4 >> SHIFT & -kHeld;  // the first group of those
    const auto ask = [&] {
#pragma unroll
      for (int o = 0; o < OUTS; ++o) {
        next_scales[o] = load_four(rs, o, next);
        if constexpr (OFFSETS) next_offsets[o] = load_four(ro, o, next);
      }
    };
    const auto multiply = [&](const i32x4 (&codes)[OUTS], int s) {
      const int g0 = (first_step + s) * 4 >> SHIFT;
      if (g0 >= next) {  // 16 more groups
        wave_meets();  // what other lanes read of the last ones
#pragma unroll
        for (int o = 0; o < OUTS; ++o) {
          T *to = held + (o * 32 + i16) * kHeldPitch + 4 * j4;
          *(Four<T> *)to = next_scales[o];
          if constexpr (OFFSETS) *(Four<T> *)(to + 16 * kHeldPitch) = next_offsets[o];
        }
        wave_meets();
        next += kHeld;
        ask();
      }
      float scale[kGroups][OUTS], offset[kGroups][OUTS];
#pragma unroll
      for (int g = 0; g < kGroups; ++g)
#pragma unroll
        for (int o = 0; o < OUTS; ++o) {
          const T *at = held + (o * 32 + i16) * kHeldPitch + g0 % kHeld + g;
          scale[g][o] = (float)at[0];
          if constexpr (OFFSETS) offset[g][o] = (float)at[16 * kHeldPitch];
        }
      bf16x8 w[4][OUTS];
#pragma unroll
      for (int o = 0; o < OUTS; ++o) {
        const i32x4 words = across_groups(codes[o]);
#pragma unroll
        for (int q = 0; q < 4; ++q) w[q][o] = numbers(words[q]);
      }
#pragma unroll
      for (int r = 0; r < TILES; ++r)
#pragma unroll
        for (int g = 0; g < kGroups; ++g) {
          const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
          f32x4 all = zero, sum[OUTS];
          if constexpr (kWhole) {
#pragma unroll
            for (int q = g << SHIFT; q < (g + 1) << SHIFT; ++q) all = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*(const bf16x8 *)(from[r] + (s * 4 + q) * 64), ones, all, 0, 0, 0);
          }
#pragma unroll
          for (int o = 0; o < OUTS; ++o) sum[o] = all;
#pragma unroll
          for (int q = g << SHIFT; q < (g + 1) << SHIFT; ++q) {
            bf16x8 x[kParts];
#pragma unroll
            for (int i = 0; i < kParts; ++i) x[i] = *(const bf16x8 *)(from[r] + (s * 4 + q) * (64 * kParts) + i * 64);
            if constexpr (kWhole) {
#pragma unroll
              for (int o = 0; o < OUTS; ++o) sum[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[0], w[q][o], sum[o], 0, 0, 0);
              continue;
            }
            f32x4 &to = OFFSETS ? all : OUTS == 1 ? sum[0] : all;
            if (!OFFSETS && OUTS > 1) all = zero;
#pragma unroll
            for (int i = kParts - 1; i >= 0; --i) to = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], ones, to, 0, 0, 0);
#pragma unroll
            for (int o = 0; o < OUTS; ++o) {
              if (!OFFSETS && OUTS > 1) sum[o] = sum[o] + all;
#pragma unroll
              for (int i = kParts - 1; i >= 0; --i) sum[o] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[i], w[q][o], sum[o], 0, 0, 0);
            }
          }
#pragma unroll
          for (int o = 0; o < OUTS; ++o)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              acc[r][o][e] = fmaf(scale[g][o], sum[o][e], acc[r][o][e]);
              if constexpr (OFFSETS) acc[r][o][e] = fmaf(offset[g][o], all[e], acc[r][o][e]);
            }
        }
    };
    if (s0 < s1) {
      Codes codes[AHEAD + 1];
      ask();
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) load(codes[i], s0 + i * STEPS);
#pragma unroll 1
      for (int s = s0; s < s1; s += STEPS) {
        load(codes[AHEAD], s + AHEAD * STEPS);
#pragma unroll
        for (int u = 0; u < STEPS; ++u)
          if (s + u < s1) multiply(codes[0].of[u], s + u);
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) codes[i] = codes[i + 1];
      }
    }
    if (TILES == 1 && p.parts > 1) {
      f32x4 *room = (f32x4 *)wave_room[wave];
      wave_meets();  // its scales have been read
      room[lane] = acc[0][0];
      __syncthreads();
      if (part == 0)
        for (int w = 1; w < p.parts; ++w) acc[0][0] += *(f32x4 *)(wave_room[wave + w] + lane * 16);
      __syncthreads();  // before the next turn's scales take the place
    }
    if (part == 0)
#pragma unroll
      for (int r = 0; r < TILES; ++r)
#pragma unroll
        for (int o = 0; o < OUTS; ++o)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int t = r * 16 + 4 * j4 + e;
            if (t >= p.rows || o * 16 + i16 >= there) continue;
            const int64_t v = first + o * 16 + i16;
            if (p.slabs)
              p.slabs[((int64_t)blockIdx.y * p.rows + t) * p.ld_slab + v] = acc[r][o][e];
            else
              p.out[t * p.ldo + v] = (T)acc[r][o][e];
          }
  }
}

// How few rows are gone over.
struct FewPlan {
  int tiles, parts, slice, slices;
  bool half;  // x takes half of a CU's LDS
  template <class T>
  void of(int64_t rows, int64_t outputs, int64_t n) {
    const int64_t steps = ceil_div(n, kStep), per_step = rows * (kStep * 2 * kPartsOf<T>);
    tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
    half = tiles == 1 && rows * 16 + steps * per_step <= Half::kStage<T>;
    const int64_t room = half ? Half::kStage<T> : tiles == 1 ? Whole::kStage<T> : Two::kStage<T>;
    int64_t k = ceil_div(steps, (room - rows * 16) / per_step);
    const int64_t outs = ceil_div(outputs, tiles == 1 ? 16 : 32);
    // as many waves as a CU takes share an output's k, or, past 16 rows, slices of it
    if (tiles > 1)
      while (outs * k < 8 * kCus && k * 4 <= steps) k *= 2;
    slice = (int)ceil_div(steps, k);
    slices = (int)ceil_div(steps, slice);
    parts = 1;
    if (tiles == 1)
      while (parts < (half ? Half::kWaves : Whole::kWaves) && outs * slices * parts < 16 * kCus && parts * 2 <= slice) parts *= 2;
  }
  FewPlan(int64_t rows, int64_t outputs, int64_t n, int32_t dtype) {
    if (dtype == SDNN_BF16)
      of<__bf16>(rows, outputs, n);
    else
      of<float>(rows, outputs, n);
  }
};
static_assert(Two::kStage<float> == FourTiles::kStage<float> && Two::kStage<__bf16> == FourTiles::kStage<__bf16>, "one room in FewPlan");

template <class S, class T>
sdnn_status launch_few(const Few<T> &p, const FewPlan &plan, int group, hipStream_t stream) {
  const int64_t turns = ceil_div(p.outputs, 16 * S::kOuts * (S::kWaves / p.parts));
  const dim3 grid((unsigned)std::min<int64_t>(turns, std::max(1, (plan.half ? 2 : 1) * kCus / plan.slices)), (unsigned)plan.slices);
  const auto go = [&](auto shift) {
    if (p.offsets)
      hipLaunchKernelGGL((k_few<T, shift(), true, S>), grid, dim3(64 * S::kWaves), 0, stream, p);
    else
      hipLaunchKernelGGL((k_few<T, shift(), false, S>), grid, dim3(64 * S::kWaves), 0, stream, p);
  };
  if (group == 32)
    go(std::integral_constant<int, 0>{});
  else if (group == 64)
    go(std::integral_constant<int, 1>{});
  else
    go(std::integral_constant<int, 2>{});
  sdnn_status st = launched("linear");
  if (st != SDNN_OK || plan.slices == 1) return st;
  return sum_slabs(p.slabs, plan.slices, p.ld_slab, Store<T>{p.out, p.ldo, p.rows, p.outputs, vector_rows(p.out, p.ldo)}, stream, "linear");
}

template <class T>
sdnn_status few_of(Few<T> p, const FewPlan &plan, int group, hipStream_t stream) {
  p.slice = plan.slice;
  p.parts = plan.parts;
  p.pairs = p.groups % 2 == 0 && (uintptr_t)p.scales % 4 == 0 && (uintptr_t)p.offsets % 4 == 0;
  if (plan.slices == 1) p.slabs = nullptr;
  if (plan.tiles == 1) return plan.half ? launch_few<Half>(p, plan, group, stream) : launch_few<Whole>(p, plan, group, stream);
  return plan.tiles == 2 ? launch_few<Two>(p, plan, group, stream) : launch_few<FourTiles>(p, plan, group, stream);
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
  // Rows for k_few, 64 at a time. Up to 64 it is never behind (us, k_few / the weights written as values: 64 x 1000 to 1000
  // outputs 12 / 12, fp32 17 / 28; 64 x 16384 to 16384 75 / 273). Past that a second pass over the codes costs less than
  // writing the weights where these are many and go to many outputs: bf16, 128 rows: 16384 to 16384 147 / 287, 4096 to
  // 16384 53 / 66, 4096 to 4096 29 / 34, but 16384 to 1024 40 / 24; 192 rows: 4096 to 16384 78 / 74. fp32, 256 rows: 4096 to 8192
  // 134 / 201, 4096 to 4096 80 / 87.
  bool few() const { return rows <= kFewRows || (outputs >= kManyOutputs && outputs * n >= kManyWeights && rows <= kFewRows * (dtype == SDNN_BF16 ? 2 : 4)); }
  int kind() const { return dtype == SDNN_BF16 ? KIND_BF16 : std::min(rows, outputs) <= kPlain ? KIND_F32 : KIND_SPLIT; }
  int64_t ld_slab() const { return ceil_div(outputs, 4) * 4; }
  int64_t values() const { return ceil_div(n, 8) * 8; }  // of a row of weights written as values
  int64_t piece() const { return std::min(outputs, std::max<int64_t>(256, kPieceValues / values() / 256 * 256)); }
  // The product's k may be split where it has few results.
  Plan product(int64_t m) const { return plan(kind(), rows, m, n, kind() != KIND_SPLIT && rows * m <= kSplitResults ? kMaxSplits : 1, kAlong); }
  int64_t pitch() const { return kind() == KIND_SPLIT ? ceil_div(n, 32) * 128 : values() * dtype_bytes(dtype); }  // of a row of x
};

struct Space {
  char *w, *x, *split;
  int *ex, *ew;
  float *slabs;
  Space(Carver &c, const Sizes &s) {
    if (s.few()) {
      size_t most = 0;
      for (const int64_t m : {std::min(s.rows, kFewRows), s.rows % kFewRows}) {
        if (m == 0) continue;
        const FewPlan p(m, s.outputs, s.n, s.dtype);
        if (p.slices > 1) most = std::max(most, (size_t)(p.slices * m * s.ld_slab()));
      }
      slabs = c.take<float>(most);
      return;
    }
    const bool parts = s.kind() == KIND_SPLIT;
    size_t most = 0;
    for (const int64_t m : {s.piece(), s.outputs % s.piece()}) {
      if (m == 0) continue;
      const Plan p = s.product(m);
      if (p.splits > 1) most = std::max(most, (size_t)(p.splits * s.rows * (ceil_div(m, 4) * 4)));
    }
    slabs = c.take<float>(most);
    w = c.take<char>((size_t)(s.piece() * s.values() * dtype_bytes(s.dtype)));
    x = c.take<char>((size_t)(s.rows * s.pitch()));
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
  hipLaunchKernelGGL((k_dequantize<T>), grid_of(ceil_div(rows, 4), ceil_div(wide, 8)), dim3(256), 0, stream, codes, scales, offsets, __builtin_ctz(group), rows, (int)n, out, ld, (int)wide, vector_rows(out, ld));
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
      st = run_shape<KIND, false, false>(s.product(m), a, b, s.rows, m, s.n, e, stream, "linear");
    } else {
      const Store<T> e{out + v0, ldo, s.rows, m, vector_rows(out + v0, ldo)};
      const Plan p = s.product(m);
      if (p.splits == 1) {
        st = run_shape<KIND, false, false>(p, a, b, s.rows, m, s.n, e, stream, "linear");
      } else {
        const int64_t ld_slab = ceil_div(m, 4) * 4;
        st = run_shape<KIND, false, false>(p, a, b, s.rows, m, s.n, Accumulate{sp.slabs, ld_slab, s.rows, m, false}, stream, "linear");
        if (st == SDNN_OK) st = sum_slabs(sp.slabs, p.splits, ld_slab, e, stream, "linear");
      }
    }
  }
  return st;
}

template <class T>
sdnn_status linear(const Sizes &s, const void *x, int64_t ldx, const uint8_t *codes, const void *scales, const void *offsets, int group, void *out, int64_t ldo, void *workspace, hipStream_t stream) {
  Carver c{(char *)workspace};
  const Space sp(c, s);
  if (s.few()) {
    for (int64_t r = 0; r < s.rows; r += kFewRows) {
      const int m = (int)std::min(s.rows - r, kFewRows);
      const Few<T> p{(const T *)x + r * ldx, ldx, aligned16(x, ldx, sizeof(T)), m, (int)s.n, codes, (const T *)scales, (const T *)offsets, (int)groups_of(s.n, group), (int)pitch_of(s.n, group),
                     s.outputs, (T *)out + r * ldo, ldo, sp.slabs, s.ld_slab(), 0, false, 1};
      const sdnn_status st = few_of<T>(p, FewPlan(m, s.outputs, s.n, s.dtype), group, stream);
      if (st != SDNN_OK) return st;
    }
    return SDNN_OK;
  }
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
