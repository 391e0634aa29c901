// Blocks of 128 x 128 outputs of fp32 operands in three bf16 parts each, whose parts all lie in LDS at once.
//
// tile.h's blocks take one part of each operand a slab: six slabs bring 12 parts of 64 values of k, of which 6 are different. Here a
// step of 32 values brings those 6 alone, and its six products are taken from registers: half the bytes from L2 and LDS. 48 KB
// a step, three steps on their way; 8 waves of 64 x 32 outputs read a step's fragments while they multiply the last one's.
// Bound by the matrix instructions and by what LDS gives beside them, about half of each's rate. The gradient's products of
// 1021 x 1000 to 2047 take 46 and 45 us so, 68 and 73 in tile.h's blocks of the same size.
#ifndef SDNN_PARTS_H
#define SDNN_PARTS_H

#include "dense.h"

namespace parts {

using namespace dense;
using tile::i32x4;

constexpr int kSide = 128, kStep = 32, kThreads = 512;
constexpr int kPart = kSide * kStep * 2;  // bytes of a part of an operand's step: 16 a lane
// Microseconds of a step in the model that chooses between these blocks and tile.h's. A step takes 1.1 to 1.2 where every CU has a
// block, but that model's figures for tile.h's are too short for three parts as well. The gradient with 0.8, with 1.0 and with 1.3, and with
// tile.h's blocks alone, us: 310 x 300 to 2000 42 / 47 / 47 / 47, 400 x 4096 to 8192 734 / 743 / 748 / 776, 2000 x 2048 to 4096
// 642 / 638 / 661 / 678, 4096 x 4096 to 8192 4955 / 4956 / 5070 / 5060; with blocks of this kind for everything 600 x 600 to 600
// takes 82 instead of 49.
constexpr double kStepUs = 0.8;

// Moves a step of one operand to LDS, a part at a time. along: rows of 64 bytes, their four chunks permuted by the row; across: 32 rows
// of k of 256 bytes, as tile::Loader lays them. Reads past the operand and past step `end` are zeros.
template <bool ACROSS, bool TWO>
struct Loader {
  uint32_t offset, offset_second;
  int chunk;
  __device__ __forceinline__ void init(const tile::Operand &op) {
    const int t = threadIdx.x, row = ACROSS ? t / 16 : t / 4;
    chunk = ACROSS ? t % 16 ^ (row << 1 & 6) : t % 4 ^ (row >> 1 & 3);
    const bool out = ACROSS && chunk * 16 >= op.extent;
    const int place = ACROSS ? tile::place3(chunk * 16) : chunk * 16;
    offset = out ? tile::kOut : row * op.pitch + place;
    if (TWO) offset_second = out ? tile::kOut : row * op.pitch_second + place;
  }
  __device__ __forceinline__ void load(const tile::Operand &op, int s, int end, int lds) const {
    uint32_t off = offset;
    uint64_t origin = (uint64_t)op.base;
    int pitch = op.pitch, rows, wide;
    if (ACROSS) {
      wide = tile::place3(min(op.extent, kSide * 2) - 1) + 1;
      rows = min((TWO && s < op.units ? min(op.first_rows, op.rows) : op.rows) - s * kStep, kStep);
      if (TWO && s >= op.units) {
        off = offset_second;
        origin = (uint64_t)op.second;
        pitch = op.pitch_second;
      }
      origin += (uint64_t)(uint32_t)(TWO && s >= op.units ? s - op.units : s) * (uint32_t)(kStep * pitch);
    } else {
      wide = min(op.extent - s * (kStep * 2), kStep * 2);
      rows = wide > 0 ? min(op.rows, kSide) : 0;
      origin += (uint64_t)(uint32_t)(s / 2) * tile::kGroup3 + s % 2 * (kStep * 2);
      if (chunk * 16 >= wide) off = tile::kOut;
    }
    if (s >= end) rows = 0;
    const int size = rows > 0 ? (rows - 1) * pitch + wide : 0;
#pragma unroll
    for (int p = 0; p < 3; ++p)
      tile::load_to_lds(i32x4{tile::uniform((int)(origin + p * tile::kSlab)), tile::uniform((int)((origin + p * tile::kSlab) >> 32)), tile::uniform(size), 0x00027000}, off, 0, lds + p * kPart);
  }
};

// Fragment addresses: subtile `i` of the wave's rows or columns from `first` on, all of the step's k.
template <bool ACROSS>
struct Reader {
  tile::Reader<tile::KIND_BF16, kSide, true> across;
  int at;
  __device__ __forceinline__ void init(int first) {
    const int lane = threadIdx.x & 63, i = lane & 15, j = lane >> 4;
    if (ACROSS)
      across.init(first);
    else
      at = (first + i) * (kStep * 2) + (j ^ (i >> 1 & 3)) * 16;
  }
  __device__ __forceinline__ i32x4 read(const char *lds, int i) const {
    if constexpr (ACROSS)
      return across.read(lds, i, 0);
    else
      return *(const i32x4 *)(lds + at + i * (16 * kStep * 2));
  }
};

template <bool ACROSS_A, bool ACROSS_B, bool TWO_B>
struct Block {
  static_assert(ACROSS_B || !TWO_B, "two matrices follow each other along k, which is across");
  static constexpr int kThreads = parts::kThreads, kTM = 4, kTN = 2, kStages = 3, kStage = 6 * kPart, kLds = kStages * kStage;
  f32x4 acc[kTM][kTN];
  static __device__ __forceinline__ int wave() { return tile::uniform(threadIdx.x >> 6); }
  static __device__ __forceinline__ int row0() { return wave() / 4 * 64; }
  static __device__ __forceinline__ int col0() { return wave() % 4 * 32; }
  static __device__ __forceinline__ bool holds() { return true; }

  struct Fragments {
    i32x4 a[3][kTM], b[3][kTN];
  };
  // Steps [s0, s1) of the operands.
  __device__ __forceinline__ void run(const tile::Operand &a, tile::Operand b, int s0, int s1, char *lds) {
    b.units *= 64 / kStep;
#pragma unroll
    for (int i = 0; i < kTM; ++i)
#pragma unroll
      for (int j = 0; j < kTN; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (s0 >= s1) return;
    Loader<ACROSS_A, false> la;
    Loader<ACROSS_B, TWO_B> lb;
    la.init(a);
    lb.init(b);
    Reader<ACROSS_A> ra;
    Reader<ACROSS_B> rb;
    ra.init(row0());
    rb.init(col0());
    const int mine = tile::uniform((int)(uintptr_t)(tile::lds_char *)lds) + wave() * 1024;
    const auto load = [&](int s, int at) {
      la.load(a, s, s1, mine + at * kStage);
      lb.load(b, s, s1, mine + at * kStage + 3 * kPart);
    };
    const auto read = [&](Fragments &f, const char *from) {
#pragma unroll
      for (int p = 0; p < 3; ++p) {
#pragma unroll
        for (int i = 0; i < kTM; ++i) f.a[p][i] = ra.read(from + p * kPart, i);
#pragma unroll
        for (int j = 0; j < kTN; ++j) f.b[p][j] = rb.read(from + (3 + p) * kPart, j);
      }
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i) load(s0 + i, i);
    tile::wait_loads<6 * (kStages - 1)>();
    tile::meet();
    Fragments even, odd;
    read(even, lds);
    int at = 0;
    const auto step = [&](int s, const Fragments &now, Fragments &next) {
      // step s + 1 has arrived, and every wave holds the fragments of step s: its buffer takes step s + 3
      tile::wait_loads<6 * (kStages - 2)>();
      tile::meet();
      const int freed = at;
      at = at + 1 == kStages ? 0 : at + 1;
      read(next, lds + at * kStage);
      load(s + kStages, freed);
      constexpr int kA[6] = {2, 0, 1, 1, 0, 0}, kB[6] = {0, 2, 1, 0, 1, 0};  // the smallest products first
#pragma unroll
      for (int p = 0; p < 6; ++p)
#pragma unroll
        for (int i = 0; i < kTM; ++i)
#pragma unroll
          for (int j = 0; j < kTN; ++j) acc[i][j] = tile::mfma<tile::KIND_BF16>(now.b[kB[p]][j], now.a[kA[p]][i], acc[i][j]);
      // a read after every one or two products (1500 x 1000 to 3000: the two products 13 us faster than in the compiler's order)
      constexpr int kReads = kTM * 3 * (ACROSS_A ? 2 : 1) + kTN * 3 * (ACROSS_B ? 2 : 1), kProducts = 6 * kTM * kTN, kEach = kProducts / kReads;
#pragma unroll
      for (int i = 0; i < kReads; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, kEach, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, kProducts - kReads * kEach, 0);
    };
#pragma unroll 1
    for (int s = s0; s < s1; s += 2) {  // (a step past s1 is zeros)
      step(s, even, odd);
      step(s + 1, odd, even);
    }
    tile::wait_loads<0>();
  }
};

// How often a product's k is split, and the time that a model of the launch gives it, as dense::plan has it.
struct Splits {
  int splits;
  double us;
};
inline Splits plan(int64_t rows, int64_t cols, int64_t k, int most_splits) {
  const int64_t blocks = ceil_div(rows, kSide) * ceil_div(cols, kSide), steps = ceil_div(k, kStep);
  Splits best = {1, 1e30};
  for (int split : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 48, 64}) {
    if (split > most_splits || (split > 1 && split * 4 > steps)) break;
    double t = (double)ceil_div(blocks * split, kCus) * (kStepUs * (double)ceil_div(steps, split) + 5.0);
    if (split > 1) t += 5.0 + 2e-6 * rows * cols * split;
    if (t < best.us) best = {split, t};
  }
  return best;
}

template <bool ACROSS_A, bool ACROSS_B, bool TWO_B, class Epilogue, class Tail = NoTail>
sdnn_status launch(const Matrix &a, const Matrix &b, int64_t rows, int64_t cols, int64_t k, int splits, const Epilogue &e, hipStream_t stream, const char *what, const Tail &tail = {}) {
  using B = Block<ACROSS_A, ACROSS_B, TWO_B>;
  Blocks blocks{};
  blocks.slabs = (int)ceil_div(k, kStep);
  blocks.per = (int)ceil_div(blocks.slabs, splits);
  blocks.splits = splits;
  blocks.rows = (int)ceil_div(rows, kSide);
  blocks.cols = (int)ceil_div(cols, kSide);
  const int64_t n = (int64_t)blocks.rows * blocks.cols * splits + tail.blocks();
  if (n * B::kThreads > 0xffffffffll || a.pitch > kMaxPitch || b.pitch > kMaxPitch || b.pitch_second > kMaxPitch) return fail(SDNN_EINVAL, "%s: %lld x %lld outputs are too many for one launch", what, (long long)rows, (long long)cols);
  hipLaunchKernelGGL((k_product<B, tile::KIND_THREE, kSide, kSide, ACROSS_A, ACROSS_B, TWO_B, Epilogue, Tail>), dim3((unsigned)n), dim3(B::kThreads), 0, stream, a, b, blocks, e, tail);
  return launched(what);
}

}  // namespace parts

#endif  // SDNN_PARTS_H
