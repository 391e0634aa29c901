// Matrix-core tile product shared by the readout's kernels: acc[m][n] = sum_k A[m][k] B[n][k] for a block of
// BM x BN outputs.
//
// Five kinds of operands share one geometry, a slab of 128 bytes of every row of A and B at a time:
//   KIND_BF16   64 bf16 values a slab.
//   KIND_SPLIT  32 fp32 values a slab, each held as two fp16 numbers whose sum it is to 22 bits or more: 64 bytes
//               of high parts, then 64 bytes of low parts. Three products (low*high, high*low, high*high) into one
//               fp32 accumulator leave out low*low, 2^-24 of a term, so that a sum is as exact as fp32
//               operands give it, at a third of the fp16 matrix rate (the fp32 matrix instructions run at a
//               sixteenth of it).
//   KIND_MX     256 4-bit values a slab with one power-of-two scale per 32 (see mx.hip).
//   KIND_THREE  64 fp32 values a group, each held as three bf16 numbers whose sum it is exactly (24 bits, at any
//               size down to 2^-110: no scale): 128 bytes of high, of middle and of low parts. A group is six slabs, one
//               for each product of parts that reaches 2^-24 of a term, each a slab of KIND_BF16; for products whose terms
//               differ so much in size that no common power of two keeps two fp16 parts of all of them.
//   KIND_F32    32 fp32 values a slab as they are, on the fp32 matrix instructions: exact products at a sixteenth of
//               the bf16 rate, for products that memory bounds and whose operands are not worth writing in two parts.
//
// An operand is "along" (rows of k: k is contiguous, 128 bytes of each row make the slab) or "across" (rows are k:
// the slab is 64 or 32 rows of BM or BN values, read from LDS through the transposing reads).
//
// Slabs go from global memory straight to LDS (16 bytes a lane), two buffers: slab s + 1 is in flight while slab s
// is multiplied. Reads past an operand's end return zeros (buffer loads with the operand's size), so ragged edges
// cost no branch and no value outside an operand is ever multiplied. LDS holds each row's 16-byte chunks
// permuted by the row number, which spreads the fragment reads over all banks.
#ifndef SDNN_TILE_H
#define SDNN_TILE_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tile {

enum Kind { KIND_BF16 = 0, KIND_SPLIT = 1, KIND_MX = 2, KIND_F32 = 3, KIND_THREE = 4 };

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kSlab = 128;             // bytes of k per row and slab
constexpr uint32_t kOut = 0x7fffff00;  // an offset past every operand: reads zeros

// One operand of a block. along: `base` is the block's first row, `rows` its rows inside the operand,
// `extent` the bytes of k. across: `base` is the block's first column, `rows` the rows of k, `extent` the
// bytes of columns inside the operand. `pitch`: bytes from row to row; 4-byte aligned, as are base
// and an along extent.
// 256 pitches stay under 2^31 (checked on the host).
// KIND_MX: `scales` is the first row's scale bytes, pitch / 16 of them a row.
// KIND_THREE: `extent` counts the bytes of one part; across, `base` is the group that holds the first column, `start`
// that column's bytes within it.
struct Operand {
  const char *base;
  int pitch, rows, extent;
  const char *scales = nullptr;
  int start = 0;
  int end = 0, parts = 0;  // KIND_THREE, set by Block: the first slab that is left out, the part of each of a group's slabs
  // An operand of two matrices (Loader's TWO). along: the block's rows are 16 of the first and 16 of the second in turn, `rows`
  // those of each. across: `units` slabs' rows of k are the first's, `first_rows` of them there, what follows the second's;
  // `rows` counts both with the first's padded to whole slabs.
  const char *second = nullptr;
  int pitch_second = 0, units = 0, first_rows = 0;
};

// Values of k that kSlabs slabs take, bytes per value of an across operand.
template <int KIND>
struct Geometry {
  static constexpr int kPerSlab = KIND == KIND_BF16 || KIND == KIND_THREE ? 64 : KIND == KIND_MX ? 256 : 32;
  static constexpr int kSlabs = KIND == KIND_THREE ? 6 : 1;
  static constexpr int kBytes = KIND == KIND_BF16 || KIND == KIND_THREE ? 2 : 4;
};

// KIND_THREE: where byte `b` of a row's high parts lies, a group's bytes, and the parts of A and of B (0 high, 1 middle, 2
// low; two bits a slab) in the order of the slabs: the smallest products first.
constexpr int kGroup3 = 3 * kSlab, kPartsA = 2 | 0 << 2 | 1 << 4 | 1 << 6 | 0 << 8 | 0 << 10, kPartsB = 0 | 2 << 2 | 1 << 4 | 0 << 6 | 1 << 8 | 0 << 10;
__host__ __device__ constexpr int place3(int b) { return b / kSlab * kGroup3 + b % kSlab; }

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// 16 bytes a lane from a buffer to LDS at `lds` + 16 * lane. Written out so that the compiler does not wait for it at
// the next LDS read: Block counts these loads itself. It has no output register; its data goes to LDS alone.
__device__ __forceinline__ void load_to_lds(i32x4 buffer, uint32_t offset, int base, int lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(base) : "memory");
}

// The same of 4 bytes a lane.
__device__ __forceinline__ void load_word_to_lds(i32x4 buffer, uint32_t offset, int base, int lds) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, %3 offen lds" ::"s"(lds), "v"(offset), "s"(buffer), "s"(base) : "memory");
}

template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "the counter's width");
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Every wave's LDS reads are done and its counted loads have arrived: from here on the others see them.
__device__ __forceinline__ void meet() {
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Moves slab `s` of one operand to LDS. ROWS: the block's rows (along) or columns (across) of this operand. TWO: they
// are two matrices' (see Operand). along, a wave loads 8 rows at once, the same of every 32 in each of its rounds, and so reads one
// of the two; across, a slab is of one.
template <int KIND, int ROWS, bool ACROSS, int THREADS, bool TWO = false>
struct Loader {
  static constexpr int kData = ROWS * kSlab;
  static constexpr int kRound = THREADS * 16;  // bytes that the workgroup moves at once
  static constexpr int kRounds = (kData + kRound - 1) / kRound;
  static constexpr int kBytes = kRounds * kRound;  // in LDS: lanes past a short slab read zeros into padding
  static constexpr int kRowBytes = ACROSS ? ROWS * Geometry<KIND>::kBytes : kSlab;  // a row in LDS
  static constexpr int kRowsPerRound = kRound / kRowBytes;
  static constexpr int kSlabRows = kData / kRowBytes;
  static_assert(kData % kRound == 0 || kRounds == 1, "whole rounds");
  static_assert(kRound % kRowBytes == 0 && kRowsPerRound % (ACROSS ? KIND == KIND_F32 ? 1 : 4 : 8) == 0, "the permutation repeats every round");

  // chunk bits that an across row's number permutes (fp32 columns are read value by value and stay)
  static constexpr int kTurn = KIND == KIND_F32 ? 0 : (kRowBytes / 16 - 1) & 6;

  static constexpr bool kTurns = TWO && !ACROSS;  // rows of two matrices in turn
  static_assert(!kTurns || (kRowsPerRound % 32 == 0 && ROWS % 32 == 0), "a wave's rows are of one matrix in every round");

  uint32_t offset;  // this lane's bytes from the slab's origin
  uint32_t offset_second;
  int chunk;        // its 16-byte chunk within the row
  int row;

  __device__ __forceinline__ void init(const Operand &op) {
    const int t = threadIdx.x % THREADS;
    row = t / (kRowBytes / 16);
    const int c = t % (kRowBytes / 16);
    chunk = ACROSS ? c ^ ((row << 1) & kTurn) : c ^ (row & 7);
    const int from = op.start + chunk * 16;  // (start is 0 but for KIND_THREE)
    const int place = ACROSS && KIND == KIND_THREE ? place3(from) : from;
    const bool out = (ACROSS && from >= op.extent) || row * kRowBytes >= kData;
    const int r = kTurns ? row / 32 * 16 + row % 16 : row;
    offset = out ? kOut : r * op.pitch + place;
    if constexpr (TWO) offset_second = out ? kOut : r * op.pitch_second + place;
  }

  // A slab's loads, issued one at a time. Past the operand's k they read zeros: every slab has kRounds of them, which the
  // waits count on.
  struct Slab {
    i32x4 buffer;
    uint32_t off;
    int step, lds;
    __device__ __forceinline__ void issue(int i) const { load_to_lds(buffer, off, i * step, lds + i * kRound); }
  };
  __device__ __forceinline__ Slab slab(const Operand &op, int s, int lds) const {
    uint32_t off = offset;
    int wide, rows, pitch = op.pitch;
    uint64_t origin = (uint64_t)op.base;
    int unit = s / Geometry<KIND>::kSlabs;  // of k
    const int within = s - unit * Geometry<KIND>::kSlabs;
    bool second = false;
    if constexpr (TWO) {
      second = kTurns ? uniform(row >> 4 & 1) : unit >= op.units;
      if (second) {
        off = offset_second;
        pitch = op.pitch_second;
        origin = (uint64_t)op.second;
      }
    }
    if (ACROSS) {
      wide = min(op.extent, op.start + kRowBytes);
      if (KIND == KIND_THREE) wide = place3(wide - 1) + 1;
      rows = min(TWO && !second ? min(op.first_rows, op.rows) - unit * kSlabRows : op.rows - unit * kSlabRows, kSlabRows);
      if (TWO && second) unit -= op.units;
      origin += (uint64_t)(uint32_t)unit * (uint32_t)(kSlabRows * pitch);
    } else {
      wide = min(op.extent - unit * kSlab, kSlab);
      rows = wide > 0 ? min(op.rows, kTurns ? ROWS / 2 : ROWS) : 0;
      origin += (uint64_t)(uint32_t)unit * (KIND == KIND_THREE ? kGroup3 : kSlab);
      if (chunk * 16 >= wide) off = kOut;
    }
    if constexpr (KIND == KIND_THREE) {
      origin += (op.parts >> 2 * within & 3) * kSlab;
      if (s >= op.end) rows = 0;
    }
    const int size = max(rows, 0) * pitch - pitch + wide;
    return {{uniform((int)origin), uniform((int)(origin >> 32)), uniform(rows > 0 ? size : 0), 0x00027000}, off, (kTurns ? kRowsPerRound / 2 : kRowsPerRound) * pitch, lds};
  }
  __device__ __forceinline__ void load(const Operand &op, int s, int lds) const {
    const Slab part = slab(op, s, lds);
#pragma unroll
    for (int i = 0; i < kRounds; ++i) part.issue(i);
  }
};

// The same for the scale bytes of KIND_MX: 8 a row and slab. Lanes past the rows read zeros into padding.
template <int ROWS, int THREADS>
struct ScaleLoader {
  static constexpr int kRound = THREADS * 4;
  static constexpr int kRounds = (ROWS * 8 + kRound - 1) / kRound;
  static constexpr int kBytes = kRounds * kRound;
  static constexpr int kRowsPerRound = kRound / 8;
  uint32_t offset;
  int half;  // of the slab's 8 bytes

  __device__ __forceinline__ void init(const Operand &op) {
    const int row = threadIdx.x % THREADS >> 1;
    half = threadIdx.x & 1;
    offset = row < ROWS ? row * (op.pitch / 16) + half * 4 : kOut;
  }
  __device__ __forceinline__ void load(const Operand &op, int s, int lds) const {
    const int wide = min(op.extent / 16 - s * 8, 8), pitch = op.pitch / 16, rows = wide > 0 ? min(op.rows, ROWS) : 0;
    const uint64_t origin = (uint64_t)op.scales + (uint64_t)(uint32_t)s * 8;
    const i32x4 r = {uniform((int)origin), uniform((int)(origin >> 32)), uniform(rows > 0 ? (rows - 1) * pitch + wide : 0), 0x00027000};
    const uint32_t off = half * 4 < wide ? offset : kOut;
    // a wave's 256 bytes follow the wave before it, as its 1024 bytes of values do
#pragma unroll
    for (int i = 0; i < kRounds; ++i) load_word_to_lds(r, off, i * kRowsPerRound * pitch, lds + i * kRound);
  }
};

// Fragment addresses of one operand: subtile `i` holds 16 rows (or columns) of the wave's part, half `q` of the slab.
// A lane gets the k values 8 (lane / 16) .. + 7 of the half (16 bytes) of row lane % 16.
template <int KIND, int ROWS, bool ACROSS>
struct Reader {
  static constexpr int kRowBytes = ACROSS ? ROWS * Geometry<KIND>::kBytes : kSlab;
  static constexpr int kTurn = (kRowBytes / 32 - 1) & 3;
  int at[ACROSS ? 4 : 2];

  // `first`: the wave's first row or column within the block: a multiple of 16, across of 32, and of 64 where the
  // wave's part is wider than 32.
  __device__ __forceinline__ void init(int first) {
    const int lane = threadIdx.x & 63, i = lane & 15, j = lane >> 4;
    if constexpr (ACROSS && KIND == KIND_F32) {
      // group j takes rows of k 4 j ... 4 j + 3, as it does of an along row's 16-byte chunk
      at[0] = 4 * j * kRowBytes + (first + i) * 4;
    } else if (ACROSS) {
      // lane i of 16 points at row i / 4 of four rows of k, 8 bytes (4 columns) at i % 4; after the
      // transposing read it holds column i of the four rows
      const int r = i >> 2;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        int granule;  // 32 bytes: 16 columns' values of one part
        if (KIND == KIND_SPLIT) {
          // columns in groups of 32: 64 bytes of high parts, 64 bytes of low ones; x = 2 * (column pair) + part
          granule = (first / 32) * 4 + x;
        } else {
          granule = first / 16 + x;
        }
        at[x] = (8 * j + r) * kRowBytes + ((granule ^ (r & kTurn)) * 32) + (i & 3) * 8;
      }
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        // 4-bit values: a lane group's two halves lie side by side, as do their scales
        const int c = KIND == KIND_MX ? 2 * j + q : 4 * q + j;
        at[q] = (first + i) * kSlab + ((c ^ (i & 7)) * 16);
      }
    }
  }

  // along: half q of subtile i. KIND_SPLIT: q is the part (0 high, 1 low).
  // across, KIND_BF16: half q of subtile i. across, KIND_SPLIT: part q of subtile i.
  __device__ __forceinline__ i32x4 read(const char *lds, int i, int q) const {
    if constexpr (!ACROSS) {
      return *(const i32x4 *)(lds + at[q] + i * (16 * kSlab));
    } else if constexpr (KIND == KIND_F32) {
      i32x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = *(const int *)(lds + at[0] + (16 * q + e) * kRowBytes + i * 64);
      return v;
    } else {
      int a;
      if constexpr (KIND == KIND_SPLIT) {
        // subtiles of 16 columns: pair i / 2 of 32 columns is 128 bytes; within it granule 2 part + i % 2
        a = at[2 * q + (i & 1)] + (i >> 1) * 128;
      } else {
        a = at[i & 3] + (i >> 2) * 128 + q * 32 * kRowBytes;
      }
      typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
      const i16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + a));
      const i16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)(lds + a + 4 * kRowBytes));
      union {
        i16x4 h[2];
        i32x4 w;
      } both = {{u, v}};
      return both.w;
    }
  }
};

// 4-bit floats (format 4, which fill half of the operand's registers), scale byte Q of the lanes' words.
template <int Q>
__device__ __forceinline__ f32x4 mfma_mx(i32x4 a, i32x4 b, f32x4 c, int scale_a, int scale_b) {
  const i32x8 wa = {a[0], a[1], a[2], a[3], 0, 0, 0, 0}, wb = {b[0], b[1], b[2], b[3], 0, 0, 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wa, wb, c, 4, 4, Q, scale_a, Q, scale_b);
}

template <int KIND>
__device__ __forceinline__ f32x4 mfma(i32x4 a, i32x4 b, f32x4 c) {
  if constexpr (KIND == KIND_F32) {
    // value e of every lane group's four: k = 4 j + e
    const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], c, 0, 0, 0);
    return c;
  } else if constexpr (KIND == KIND_BF16 || KIND == KIND_THREE)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The product of one block. WM x WN waves share it, each BM / WM x BN / WN outputs in subtiles of 16 x 16.
// acc[i][j]: rows 16 i + lane % 16 of the wave's part, columns 16 j + 4 (lane / 16) + 0..3.
//
// STAGES buffers in LDS. A slab is multiplied in passes: its two halves (bf16, three parts, 4-bit), or high*high, high*low, low*high
// (KIND_SPLIT). A pass goes down the subtiles of A, and each one's registers take the next pass's fragment as soon as
// its products are issued, so that LDS reads run between products and one set of A fragments is enough. A little
// into a slab's last pass, when its last fragments have been read, the waves meet, and the slab's buffer takes
// slab s + STAGES: its loads have a slab's time.
//
// 256 x 256 by 8 waves of 128 x 64: two waves a SIMD cover each other's waits, and 208 of 256 registers hold sums and
// fragments. Measured on 8192^3: bf16 1300 TFLOP/s at 66% of the cycles in matrix instructions (the card lowers its
// clock to 1.9 GHz under them; the library's kernel in the same run 1570), KIND_SPLIT 1430, 477 of fp32.
// Four waves of 128 x 128 read less LDS and measured 1010, raised wave priorities during the products 7% less.
//
// GROUPS of WM x WN waves may share the block's outputs, each loading and taking every GROUPS-th slab, with their sums joined
// through LDS at the end: a launch of few blocks runs through k in fewer meetings.
//
// TWO_B: B's rows are two matrices' (see Operand).
template <int KIND, int BM, int BN, int WM, int WN, bool ACROSS_A, bool ACROSS_B, int STAGES, int GROUPS = 1, bool TWO_B = false>
struct Block {
  static constexpr int kWaves = WM * WN, kGroup = 64 * kWaves, kThreads = kGroup * GROUPS;
  static constexpr int kTM = BM / WM / 16, kTN = BN / WN / 16;
  using LoadA = Loader<KIND, BM, ACROSS_A, kGroup>;
  using LoadB = Loader<KIND, BN, ACROSS_B, kGroup, TWO_B>;
  using ScaleA = ScaleLoader<BM, kGroup>;
  using ScaleB = ScaleLoader<BN, kGroup>;
  static constexpr bool kMx = KIND == KIND_MX;
  static constexpr bool kRagged = KIND == KIND_BF16 || KIND == KIND_F32;  // rows that are read in place may end within a chunk
  static constexpr int kValuesA = LoadA::kBytes, kValues = kValuesA + LoadB::kBytes;
  static constexpr int kPart = kValues + (kMx ? ScaleA::kBytes + ScaleB::kBytes : 0);  // a group's slab
  static constexpr int kStage = GROUPS * kPart;
  static constexpr int kLds = STAGES * kStage;
  static_assert(kLds <= 160 * 1024, "LDS of a CU");
  static constexpr int kLoads = LoadA::kRounds + LoadB::kRounds + (kMx ? ScaleA::kRounds + ScaleB::kRounds : 0);  // of a wave and stage
  static_assert(GROUPS == 1 || kStage * STAGES >= (GROUPS - 1) * BM * BN * 4, "the sums' room");

  f32x4 acc[kTM][kTN];

  __device__ __forceinline__ static int wave() { return uniform(threadIdx.x >> 6); }
  __device__ __forceinline__ static int group() { return GROUPS == 1 ? 0 : wave() / kWaves; }
  __device__ __forceinline__ static int member() { return GROUPS == 1 ? wave() : wave() % kWaves; }
  __device__ __forceinline__ static int row0() { return (member() / WN) * (BM / WM); }
  __device__ __forceinline__ static int col0() { return (member() % WN) * (BN / WN); }

  template <class R>
  __device__ __forceinline__ static void read(const R &r, const char *lds, int q, i32x4 (&f)[kTN]) {
#pragma unroll
    for (int j = 0; j < kTN; ++j) f[j] = r.read(lds, j, q);
  }
  // A subtile's scale bytes: the two of a lane's blocks.
  __device__ __forceinline__ static int read_scale(const char *lds, int first, int i) {
    const int lane = threadIdx.x & 63;
    return *(const uint16_t *)(lds + (first + 16 * i + (lane & 15)) * 8 + 2 * (lane >> 4));
  }
  template <int Q>
  __device__ __forceinline__ void multiply(int i, i32x4 a, const i32x4 (&b)[kTN], int scale, const int (&scales)[kTN]) {
#pragma unroll
    for (int j = 0; j < kTN; ++j)
      if constexpr (kMx)
        acc[i][j] = mfma_mx<Q>(b[j], a, acc[i][j], scales[j], scale);
      else
        acc[i][j] = mfma<KIND>(b[j], a, acc[i][j]);
  }
  // Nothing of the operand past slab s1.
  __device__ __forceinline__ static void clip(Operand &op, bool across, int slab_rows, int s1) {
    if constexpr (KIND == KIND_THREE) {
      op.end = uniform(s1);
      op.start = uniform(op.start);
    } else {
      int &k = across ? op.rows : op.extent;
      const int64_t end = (int64_t)s1 * (across ? slab_rows : kSlab);
      if (end < k) k = (int)end;
    }
    op.pitch = uniform(op.pitch);
    op.rows = uniform(op.rows);
    op.extent = uniform(op.extent);
    op.pitch_second = uniform(op.pitch_second);
  }

  // The last slab of rows that end within a 16-byte chunk holds what follows them there: zeros take its place.
  template <int ROWS, int THREADS>
  __device__ __forceinline__ static void trim(char *lds, int extent) {
    const int chunk = (extent % kSlab) / 16, first = extent % 16 / 4;
    for (int r = threadIdx.x % THREADS; r < ROWS; r += THREADS)
      for (int i = first; i < 4; ++i) *(int *)(lds + r * kSlab + ((chunk ^ (r & 7)) * 16) + i * 4) = 0;
  }

  // The order that the scheduler is to keep: products and LDS reads as they are written.
  template <int SUBTILES>
  __device__ __forceinline__ static void products() {
    if constexpr (SUBTILES > 0) __builtin_amdgcn_sched_group_barrier(0x008, SUBTILES * kTN * (KIND == KIND_F32 ? 4 : 1), 0);
  }
  template <int READS>
  __device__ __forceinline__ static void reads() {
    if constexpr (READS > 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }

  // Slabs [s0, s1) of the operands.
  __device__ __forceinline__ void run(Operand a, Operand b, int s0, int s1, char *lds) {
    clip(a, ACROSS_A, LoadA::kSlabRows, s1);
    clip(b, ACROSS_B, LoadB::kSlabRows, s1);
    a.parts = kPartsA;
    b.parts = kPartsB;
    LoadA la;
    LoadB lb;
    ScaleA lsa;
    ScaleB lsb;
    la.init(a);
    lb.init(b);
    if constexpr (kMx) {
      lsa.init(a);
      lsb.init(b);
    }
    Reader<KIND, BM, ACROSS_A> ra;
    Reader<KIND, BN, ACROSS_B> rb;
    ra.init(row0());
    rb.init(col0());
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
      for (int j = 0; j < kTN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (s0 >= s1) return;
    lds += group() * kPart;
    s0 += group();
    const int base = uniform((int)(uintptr_t)(lds_char *)lds), mine = base + member() * 1024;
    const auto load_scales = [&](int s, int to) {
      if constexpr (kMx) {
        const int at = base + to + kValues + member() * 256;
        lsa.load(a, s, at);
        lsb.load(b, s, at + ScaleA::kBytes);
      }
    };
    const auto load = [&](int s, int to) {
      load_scales(s, to);
      la.load(a, s, mine + to);
      lb.load(b, s, mine + to + kValuesA);
    };
#pragma unroll
    for (int i = 0; i < STAGES; ++i) load(s0 + i * GROUPS, i * kStage);
    wait_loads<(STAGES - 1) * kLoads>();
    meet();
    const bool ragged_a = !ACROSS_A && (a.extent & 15), ragged_b = !ACROSS_B && (b.extent & 15);
    const auto trim_last = [&](int s, char *stage) {
      if (!ragged_a && !ragged_b) return;
      const int s_a = (a.extent - 1) / kSlab, s_b = (b.extent - 1) / kSlab, round = s - group();
      const bool now_a = ragged_a && s_a >= round && s_a < round + GROUPS, now_b = ragged_b && s_b >= round && s_b < round + GROUPS;
      if (now_a && s_a == s) trim<BM, kGroup>(stage, a.extent);
      if (now_b && s_b == s) trim<BN, kGroup>(stage + kValuesA, b.extent);
      if (now_a || now_b) meet();
    };
    if constexpr (kRagged) trim_last(s0, lds);
    constexpr int kAcross = KIND == KIND_F32 ? 4 : 2;                      // LDS reads of a fragment across
    constexpr int kEach = kMx ? 2 : ACROSS_A ? kAcross : 1;                // with a subtile of A
    constexpr int kAll = kTN * (kMx ? 2 : ACROSS_B ? kAcross : 1);         // with all of B
    i32x4 fa[kTM], fb[kTN], gb[kTN];
    int sa[kTM], sb[kTN];
    read(rb, lds + kValuesA, 0, fb);
#pragma unroll
    for (int i = 0; i < kTM; ++i) fa[i] = ra.read(lds, i, 0);
#pragma unroll
    for (int i = 0; i < kTM; ++i) sa[i] = kMx ? read_scale(lds + kValues, row0(), i) : 0;
#pragma unroll
    for (int j = 0; j < kTN; ++j) sb[j] = kMx ? read_scale(lds + kValues + ScaleA::kBytes, col0(), j) : 0;
    int at = 0;
    for (int s = s0; s < s1 + group(); s += GROUPS) {  // as often in every group: past s1 a slab is zeros
      const int used = at * kStage;
      const char *now = lds + used;
      at = at + 1 == STAGES ? 0 : at + 1;
      const char *then = lds + at * kStage;
      read(rb, now + kValuesA, 1, gb);
      reads<kTN * (ACROSS_B ? kAcross : 1)>();
      if constexpr (KIND == KIND_SPLIT) {
#pragma unroll
        for (int i = 0; i < kTM; ++i) multiply<0>(i, fa[i], fb, 0, sb);
        products<kTM>();
      }
#pragma unroll
      for (int i = 0; i < kTM; ++i) {
        multiply<0>(i, fa[i], KIND == KIND_SPLIT ? gb : fb, sa[i], sb);
        fa[i] = ra.read(now, i, 1);
        products<1>();
        reads<ACROSS_A ? kAcross : 1>();
      }
      constexpr int kDelay = kTM < 4 ? kTM / 2 : 2;
#pragma unroll
      for (int i = 0; i < kDelay; ++i) multiply<1>(i, fa[i], KIND == KIND_SPLIT ? fb : gb, sa[i], sb);
      products<kDelay>();
#pragma unroll
      for (int i = 0; i < kDelay; ++i)
#pragma unroll
        for (int j = 0; j < kTN; ++j) asm volatile("" : "+v"(acc[i][j]));  // ahead of the meeting
      // slab s + 1 has arrived; all fragments of slab s are in registers
      wait_loads<(STAGES - 2) * kLoads>();
      meet();
      if constexpr (kRagged) trim_last(s + GROUPS, lds + at * kStage);
      constexpr bool kSpread = kTM >= 8 && GROUPS == 1;  // a small block has no time to spread its loads over
      if constexpr (kSpread)
        load_scales(s + STAGES, used);
      else
        load(s + STAGES * GROUPS, used);
      const auto next_a = la.slab(a, s + STAGES, mine + used);
      const auto next_b = lb.slab(b, s + STAGES, mine + used + kValuesA);
      constexpr int kValueLoads = LoadA::kRounds + LoadB::kRounds;
      int issued = 0;
      const auto issue = [&](int until) {
#pragma unroll
        for (int i = 0; i < kValueLoads; ++i)
          if (i >= issued && i < until) {
            if (i < LoadA::kRounds)
              next_a.issue(i);
            else
              next_b.issue(i - LoadA::kRounds);
          }
        issued = until;
      };
      i32x4 hb[kTN];
      int hs[kTN];
      read(rb, then + kValuesA, 0, hb);
#pragma unroll
      for (int j = 0; j < kTN; ++j) hs[j] = kMx ? read_scale(then + kValues + ScaleA::kBytes, col0(), j) : 0;
#pragma unroll
      for (int i = 0; i < kDelay; ++i) {
        fa[i] = ra.read(then, i, 0);
        if (kMx) sa[i] = read_scale(then + kValues, row0(), i);
      }
      reads<kAll + kDelay * kEach>();
#pragma unroll
      for (int i = kDelay; i < kTM; ++i) {
        multiply<1>(i, fa[i], KIND == KIND_SPLIT ? fb : gb, sa[i], sb);
        fa[i] = ra.read(then, i, 0);
        if (kMx) sa[i] = read_scale(then + kValues, row0(), i);
        if constexpr (kSpread) issue(kValueLoads * (i - kDelay + 1) / (kTM - kDelay));
        products<1>();
        reads<kEach>();
      }
#pragma unroll
      for (int j = 0; j < kTN; ++j) {
        fb[j] = hb[j];
        sb[j] = hs[j];
      }
    }
    wait_loads<0>();
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
      for (int j = 0; j < kTN; ++j) asm volatile("" : "+v"(acc[i][j]));  // stays ahead of the epilogue's branches
    if constexpr (GROUPS > 1) {
      f32x4 *room = (f32x4 *)(lds - group() * kPart) + member() * (kTM * kTN * 64) + (threadIdx.x & 63);
      __syncthreads();
      if (group() > 0) {
#pragma unroll
        for (int i = 0; i < kTM * kTN; ++i) room[((group() - 1) * kWaves * kTM * kTN + i) * 64] = acc[i / kTN][i % kTN];
      }
      __syncthreads();
      if (group() == 0) {
#pragma unroll
        for (int g = 0; g < GROUPS - 1; ++g)
#pragma unroll
          for (int i = 0; i < kTM * kTN; ++i) acc[i / kTN][i % kTN] += room[(g * kWaves * kTM * kTN + i) * 64];
      }
    }
  }
  // The waves that hold the block's sums after run().
  __device__ __forceinline__ static bool holds() { return GROUPS == 1 || group() == 0; }
};

}  // namespace tile

#endif  // SDNN_TILE_H
