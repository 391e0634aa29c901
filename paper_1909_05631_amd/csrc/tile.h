// Matrix-core tile product shared by the readout's kernels: acc[m][n] = sum_k A[m][k] B[n][k] for a block of
// BM x BN outputs.
//
// Three kinds of operands share one geometry, a slab of 128 bytes of every row of A and B at a time:
//   KIND_BF16   64 bf16 values a slab.
//   KIND_SPLIT  32 fp32 values a slab, each held as two fp16 numbers whose sum it is to 22 bits or more: 64 bytes
//               of high parts, then 64 bytes of low parts. Three products (low*high, high*low, high*high) into one
//               fp32 accumulator leave out low*low, 2^-24 of a term, so that a sum is as exact as fp32
//               operands give it, at a third of the fp16 matrix rate (the fp32 matrix instructions run at a
//               sixteenth of it).
//   KIND_MX     256 4-bit values a slab with one power-of-two scale per 32 (see mx.hip).
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

enum Kind { KIND_BF16 = 0, KIND_SPLIT = 1, KIND_MX = 2 };

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

constexpr int kSlab = 128;             // bytes of k per row and slab
constexpr uint32_t kOut = 0x7fffff00;  // an offset past every operand: reads zeros

// One operand of a block. along: `base` is the block's first row, `rows` its rows inside the operand,
// `extent` the bytes of k. across: `base` is the block's first column, `rows` the rows of k, `extent` the
// bytes of columns inside the operand. `pitch`: bytes from row to row; 16-byte aligned, as is base.
// (rows of a slab) * pitch stays under 2^31 (checked on the host).
struct Operand {
  const char *base;
  int64_t pitch;
  int64_t rows;
  int64_t extent;
};

// Values per slab, bytes per value of an across operand.
template <int KIND>
struct Geometry {
  static constexpr int kPerSlab = KIND == KIND_BF16 ? 64 : KIND == KIND_SPLIT ? 32 : 256;
  static constexpr int kBytes = KIND == KIND_BF16 ? 2 : 4;
};

// Moves slab `s` of one operand to LDS. ROWS: the block's rows (along) or columns (across) of this operand.
template <int KIND, int ROWS, bool ACROSS, int THREADS>
struct Loader {
  static constexpr int kBytes = ROWS * kSlab;
  static constexpr int kRound = THREADS * 16;  // bytes that the workgroup moves at once
  static constexpr int kRounds = (kBytes + kRound - 1) / kRound;
  static constexpr int kRowBytes = ACROSS ? ROWS * Geometry<KIND>::kBytes : kSlab;  // a row in LDS
  static constexpr int kRowsPerRound = kRound / kRowBytes;
  static constexpr int kSlabRows = kBytes / kRowBytes;
  static_assert(kBytes % kRound == 0 || kRounds == 1, "whole rounds");
  static_assert(kRowBytes <= kRound || ACROSS, "a round holds whole rows");
  static_assert(!ACROSS || (kRound % kRowBytes == 0 && kRowsPerRound % 4 == 0) || kRounds == 1, "the permutation repeats every round");

  static constexpr int kTurn = (kRowBytes / 16 - 1) & 6;  // chunk bits that an across row's number permutes

  uint32_t offset;  // this lane's bytes from the slab's origin
  int chunk;        // its 16-byte chunk within the row
  int row;

  __device__ __forceinline__ void init(const Operand &op) {
    const int t = threadIdx.x;
    row = t / (kRowBytes / 16);
    const int c = t % (kRowBytes / 16);
    chunk = ACROSS ? c ^ ((row << 1) & kTurn) : c ^ (row & 7);
    offset = (uint32_t)(row * op.pitch) + chunk * 16;
    if (ACROSS && chunk * 16 >= op.extent) offset = kOut;
  }

  __device__ __forceinline__ void load(const Operand &op, int64_t s, char *lds) const {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const char *origin;
    uint32_t size, off = offset;
    if (ACROSS) {
      const int64_t left = op.rows - s * kSlabRows;
      const int n = left < kSlabRows ? (int)left : kSlabRows;
      const int wide = op.extent < kRowBytes ? (int)op.extent : kRowBytes;
      origin = op.base + s * kSlabRows * op.pitch;
      size = n > 0 ? (uint32_t)((n - 1) * op.pitch) + wide : 0;
    } else {
      const int64_t left = op.extent - s * kSlab;
      const int wide = left < kSlab ? (int)left : kSlab;
      const int n = op.rows < ROWS ? (int)op.rows : ROWS;
      origin = op.base + s * kSlab;
      size = n > 0 && wide > 0 ? (uint32_t)((n - 1) * op.pitch) + wide : 0;
      if (chunk * 16 >= wide) off = kOut;
    }
    const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc((void *)origin, 0, size, 0x00027000);
    const int step = (int)(kRowsPerRound * op.pitch);
#pragma unroll
    for (int i = 0; i < kRounds; ++i) {
      if (kBytes < kRound && wave * 1024 >= kBytes) break;
      __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_void *)(lds + i * kRound + wave * 1024), 16, off, i * step, 0, 0);
    }
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
    if (ACROSS) {
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

template <int KIND>
__device__ __forceinline__ f32x4 mfma(i32x4 a, i32x4 b, f32x4 c) {
  if constexpr (KIND == KIND_BF16)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// The product of one block. WM x WN waves share it, each BM / WM x BN / WN outputs in subtiles of 16 x 16.
// acc[i][j]: rows 16 i + lane % 16 of the wave's part, columns 16 j + 4 (lane / 16) + 0..3.
template <int KIND, int BM, int BN, int WM, int WN, bool ACROSS_A, bool ACROSS_B>
struct Block {
  static constexpr int kThreads = 64 * WM * WN;
  static constexpr int kTM = BM / WM / 16, kTN = BN / WN / 16;
  static constexpr int kStage = (BM + BN) * kSlab;
  static constexpr int kLds = 2 * kStage;
  using LoadA = Loader<KIND, BM, ACROSS_A, kThreads>;
  using LoadB = Loader<KIND, BN, ACROSS_B, kThreads>;

  f32x4 acc[kTM][kTN];

  __device__ __forceinline__ static int wave() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }
  __device__ __forceinline__ static int row0() { return (wave() / WN) * (BM / WM); }
  __device__ __forceinline__ static int col0() { return (wave() % WN) * (BN / WN); }

  // Slabs [s0, s1) of the operands.
  __device__ __forceinline__ void run(const Operand &a, const Operand &b, int64_t s0, int64_t s1, char *lds) {
    LoadA la;
    LoadB lb;
    la.init(a);
    lb.init(b);
    Reader<KIND, BM, ACROSS_A> ra;
    Reader<KIND, BN, ACROSS_B> rb;
    ra.init(row0());
    rb.init(col0());
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
      for (int j = 0; j < kTN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (s0 < s1) {
      la.load(a, s0, lds);
      lb.load(b, s0, lds + BM * kSlab);
    }
    for (int64_t s = s0; s < s1; ++s) {
      char *now = lds + ((s - s0) & 1) * kStage, *next = lds + ((s - s0 + 1) & 1) * kStage;
      // slab s has arrived, and every wave is done with the buffer that slab s + 1 goes to
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      step(ra, rb, now);
      if (s + 1 < s1) {
        la.load(a, s + 1, next);
        lb.load(b, s + 1, next + BM * kSlab);
      }
      multiply();
    }
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
      for (int j = 0; j < kTN; ++j) asm volatile("" : "+v"(acc[i][j]));  // stays ahead of the epilogue's branches
  }

  i32x4 fa[kTM][2], fb[kTN][2];

  template <class RA, class RB>
  __device__ __forceinline__ void step(const RA &ra, const RB &rb, const char *now) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
#pragma unroll
      for (int j = 0; j < kTN; ++j) fb[j][q] = rb.read(now + BM * kSlab, j, q);
#pragma unroll
      for (int i = 0; i < kTM; ++i) fa[i][q] = ra.read(now, i, q);
    }
  }

  __device__ __forceinline__ void multiply() {
    if constexpr (KIND == KIND_SPLIT) {
#pragma unroll
      for (int i = 0; i < kTM; ++i)
#pragma unroll
        for (int j = 0; j < kTN; ++j) acc[i][j] = mfma<KIND>(fb[j][0], fa[i][0], acc[i][j]);
#pragma unroll
      for (int i = 0; i < kTM; ++i)
#pragma unroll
        for (int j = 0; j < kTN; ++j) acc[i][j] = mfma<KIND>(fb[j][1], fa[i][0], acc[i][j]);
#pragma unroll
      for (int i = 0; i < kTM; ++i)
#pragma unroll
        for (int j = 0; j < kTN; ++j) acc[i][j] = mfma<KIND>(fb[j][0], fa[i][1], acc[i][j]);
    } else {
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
          for (int j = 0; j < kTN; ++j) acc[i][j] = mfma<KIND>(fb[j][q], fa[i][q], acc[i][j]);
    }
  }
};

}  // namespace tile

#endif  // SDNN_TILE_H
