// A gated hidden layer on rows of features, h = act(g) * u with g = x wg^T and u = x wu^T, and its gradient:
//
//   dg = dh * u * act'(g),  du = dh * act(g)
//   dx = dg wg + du wu,  dwg = dg^T x,  dwu = du^T x
//
// Layer: one product. A block's columns are 16 rows of wg and 16 of wu in turn, read where they are, so that a wave
// holds g and u of the same outputs in neighbouring subtiles and the epilogue takes the activation and the product from
// fp32 sums; g and u are written only where the caller keeps them for the gradient. Where there are few outputs and blocks for
// only a part of the CUs, the features are split and a second kernel joins the parts.
// Gradient: one pass over g, u and dh writes dg and du side by side, a row of 2 H values (each half padded to whole
// slabs of k with zeros). Then two products read them: dx = [dg du] [wg; wu], whose k goes through both halves into one
// sum, and [dwg; dwu] = [dg du]^T x. Nothing is transposed or concatenated in memory.
//
// fp32: the layer's sums run along rows of x and w, which take a power of two each and go in two fp16 parts; the gradient's run
// across rows of any size, so dg, du, w and x go there in three bf16 parts, which need no scale. Where rows or outputs are few
// all go to the fp32 matrix instructions as they are. Up to 16 rows have a kernel of their own (k_few_rows).
//
// What bounds it, measured on this card (a copy runs at 4.9 TB/s, the library's bf16 product at 1633 TFLOP/s):
//   8192 x 4096 to 16384, bf16: 5.45 ms, matrix instructions: the layer 1.75 ms (1260 TFLOP/s; 0.1 ms of it for keeping g and
//     u), dg and du 0.27 ms (1.34 GB at 5.0 TB/s), dx and the weights' gradients 1.6 ms each (1370).
//   2000 x 4096 to 16384, bf16, the layer alone: 433 us, 1240 TFLOP/s.
//   64 x 1024 to 4096, bf16: 35 us, four launches of 4 to 10 us, and the host's time for them.
//   1021 x 1000 to 2047, fp32: 167 us: the layer 48 us and 13 for x and w in parts, the gradient's two products 46 and 45 us in
//     three parts (185 TFLOP/s of 275: one block a CU, see parts.h), 22 us for its slopes and parts.
//   1 x 4096 to 16384, bf16: 50 us, the weights at 5.3 TB/s; 16 rows 55 us.
#include "dense.h"
#include "few.h"
#include "copies.h"
#include "parts.h"
#include "sums.h"

#include <utility>

using namespace dense;
using namespace copies;
using namespace sums;
using tile::i32x4;
using tile::KIND_BF16;
using tile::KIND_F32;
using tile::KIND_SPLIT;
using tile::KIND_THREE;

namespace {

constexpr int64_t kMaxHidden = 1 << 19;    // a row of dg and du in three parts is then the longest that the tiles take
constexpr int64_t kSplitValues = 1 << 24;  // values of g and u whose features may be split: past that there is a 256 x 256 block for every CU
// fp32 rows or outputs for the plain fp32 products, which read the operands as they are, and, for the gradient, the fewer of both
// where all three sizes' product is at most kSmall. us, plain and in parts: the layer 1000 to 2048, 64 rows 18 / 25, 192 rows 26 / 26,
// 300 rows 43 / 32, 4096 to 8192, 128 rows 147 / 211, 192 210 / 238, 300 402 / 271, 8192 x 4096 to 64 outputs 86 / 104, 96 118 / 122,
// 128 146 / 129; the gradient 1000 to 2048, 64 rows 29 / 39, 192 48 / 47, 250 54 / 53, 300 66 / 59, 4096 to 8192, 128 337 / 414, 192
// 446 / 476, 256 618 / 544, 8192 x 4096 to 64 outputs 194 / 224, 96 329 / 270; but 300 x 300 to 400 24 / 29, 2000 x 1000 to 128
// 42 / 46, to 250 61 / 55. (One border of outputs for both: the gradient's own would be 64, since it pads halves to 64 outputs.)
constexpr int64_t kPlainRows = 192, kPlainHidden = 96, kPlainSmall = 300, kSmall = 1 << 28;

// exp(x + rest), rest far smaller than x, to two units of its last place: what the exponent's rounding loses, up to 2^-17 of the
// result, is put back as a factor.
__device__ __forceinline__ float exp_of_sum(float x, float rest) {
  constexpr float kLog = 1.44269504088896340736f, kLogRest = 1.44269504088896340736 - (double)kLog;
  const float y = x * kLog, lost = fmaf(x, kLog, -y) + fmaf(x, kLogRest, rest * kLog);
  return __builtin_amdgcn_exp2f(y) * fmaf(lost, 0.69314718055994530942f, 1.0f);
}

// act(g) and, for the gradient, act'(g), for values of type T: where act goes to zero, fp32 keeps its relative precision. bf16 has
// no such bits, and takes exp as it is: off by (g^2 + 8) 2^-24 of itself there for gelu, (|g| + 8) 2^-24 for silu.
struct Activated {
  float value, slope;
};
template <class T, bool SLOPE>
__device__ __forceinline__ Activated activated(int activation, float g) {
  constexpr bool kFull = sizeof(T) == 4;
  Activated a;
  a.slope = 0.0f;
  if (activation == SDNN_SILU) {
    // g p with p = 1 / (1 + exp(-g)); the exponential may be infinite: p is then 0
    const float e = kFull ? exp_of_sum(__builtin_amdgcn_fmed3f(-g, -200.0f, 200.0f), 0.0f) : few::exp_of(-g);
    const float p = __builtin_amdgcn_rcpf(1.0f + e);  // (to one unit of its last place)
    a.value = g * p;
    if (SLOPE) a.slope = fmaf(a.value, 1.0f - p, p);
  } else if (activation == SDNN_GELU) {
    // g P with P the normal distribution, whose tail below -|g| is exp(-g^2 / 2) t p(t), t = 1 / (1 + |g| / sqrt 8): p is
    // fitted to erfc's scaled form there (9th degree, by least squares reweighted towards the largest relative error, 2e-8), so that
    // the tail is within 3.7e-7 of itself with fp32's roundings (the layer 2000 x 4096 to 16384: 456 us, with erfcf 487)
    constexpr float kTail[10] = {0.141032249f, 0.14142856f, 0.119322069f, 0.112772763f, -0.0491647162f, 0.210649297f, -0.335027367f, 0.214477479f, -0.0616335161f, 0.006143176f};
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(g), 0.35355339059327f, 1.0f));
    const float q = fminf(fabsf(g), 16.0f), square = q * q;  // (exp(-128) is zero)
    const float e = kFull ? exp_of_sum(-0.5f * square, -0.5f * fmaf(q, q, -square)) : few::exp_of(-0.5f * g * g);
    float p = kTail[9];
#pragma unroll
    for (int i = 8; i >= 0; --i) p = fmaf(p, t, kTail[i]);
    p *= t * e;
    if (g > 0.0f) p = 1.0f - p;
    a.value = g * p;
    if (SLOPE) a.slope = fmaf(g * 0.39894228040143267794f, e, p);
  } else {
    a.value = g <= 0.0f ? 0.0f : g;
    if (SLOPE) a.slope = g > 0.0f ? 1.0f : 0.0f;
  }
  return a;
}

// ------------------------------------------------------------------------------------------------
// The layer's results

template <int KIND, class T>
struct Layer {
  const int *ex, *eg, *eu;  // exponents of the rows of x, wg and wu (KIND_SPLIT)
  int activation;
  int64_t rows, hidden;
  T *h, *gate, *up;  // gate and up: nullptr where they are not kept; h: nullptr where they alone are wanted
  int64_t ldh, ldg, ldu;
  bool vec_h, vec_g, vec_u;
  // The exponents of four neighbouring outputs, from c on, and four sums of a row with exponent e without them.
  __device__ __forceinline__ i32x4 columns(const int *exponents, int64_t c) const {
    i32x4 e = {0, 0, 0, 0};
    if constexpr (KIND == KIND_SPLIT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = c + i < hidden ? exponents[c + i] : 0;
    }
    return e;
  }
  __device__ __forceinline__ f32x4 scaled(f32x4 s, int e, i32x4 columns) const {
    if constexpr (KIND == KIND_SPLIT) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = ldexpf(s[i], -e - columns[i]);
    }
    return s;
  }
  __device__ __forceinline__ f32x4 product(f32x4 g, f32x4 u) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) g[i] = activated<T, false>(activation, g[i]).value * u[i];
    return g;
  }
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
    constexpr int N = B::kTN / 2;  // pairs of subtiles: g and u
    static_assert(B::kTN % 2 == 0, "whole pairs");
    const int i16 = threadIdx.x & 15, j4 = (threadIdx.x & 63) >> 4;
    const int64_t first = col0 / 2;
    i32x4 cg[N], cu[N];  // read once for all rows
#pragma unroll
    for (int j = 0; j < N; ++j) {
      cg[j] = columns(eg, first + 16 * j + 4 * j4);
      cu[j] = columns(eu, first + 16 * j + 4 * j4);
    }
    int rows_e[B::kTM];
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) rows_e[i] = KIND == KIND_SPLIT && row0 + 16 * i + i16 < rows ? ex[row0 + 16 * i + i16] : 0;
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      const int64_t t = row0 + 16 * i + i16;
      const bool in = t < rows;
      const auto g = [&](int j) { return scaled(block.acc[i][2 * j], rows_e[i], cg[j]); };
      const auto u = [&](int j) { return scaled(block.acc[i][2 * j + 1], rows_e[i], cu[j]); };
      if (gate) store_row<T, N>(gate + t * ldg, first, hidden, vec_g, in, g);
      if (up) store_row<T, N>(up + t * ldu, first, hidden, vec_u, in, u);
      if (h) store_row<T, N>(h + t * ldh, first, hidden, vec_h, in, [&](int j) { return product(g(j), u(j)); });
    }
  }
};

// The same from sums whose k was split: slabs of 16 columns of g and 16 of u in turn, `ld` a row.
template <int KIND, class T>
__global__ __launch_bounds__(256) void k_layer_slabs(const float *slabs, int splits, int64_t ld, Layer<KIND, T> to) {
  const int64_t t = blockIdx.y;
  const int e = KIND == KIND_SPLIT ? to.ex[t] : 0;
  for (int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; c < to.hidden; c += (int64_t)gridDim.x * 1024) {
    const float *from = slabs + t * ld + c / 16 * 32 + c % 16;
    f32x4 g = {0.0f, 0.0f, 0.0f, 0.0f}, u = g;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
      g += *(const f32x4 *)(from + s * to.rows * ld);
      u += *(const f32x4 *)(from + s * to.rows * ld + 16);
    }
    g = to.scaled(g, e, to.columns(to.eg, c));
    u = to.scaled(u, e, to.columns(to.eu, c));
    const int n = to.hidden - c < 4 ? (int)(to.hidden - c) : 4;
    if (to.gate) store4(to.gate + t * to.ldg + c, g, n, to.vec_g);
    if (to.up) store4(to.up + t * to.ldu + c, u, n, to.vec_u);
    if (to.h) store4(to.h + t * to.ldh + c, to.product(g, u), n, to.vec_h);
  }
}

// ------------------------------------------------------------------------------------------------
// The layer of few rows

// Up to 16 rows of x stay in LDS while the weights stream past, each byte once, from memory to registers to the matrix
// instructions: 16 outputs of a wave at a time, their rows of wg and of wu, 128 bytes of each row a step. Waves in teams of
// `parts` share an output's k. Bound by the weights' bytes; the tiles would go through k in a few long chains.
constexpr int kStepBytes = 128;

template <int KIND, class T>
struct FewRows {
  const T *x;
  int64_t ldx;
  bool vec_x;
  int rows, n;
  const char *wg, *wu;
  int pitch_g, pitch_u;  // bytes
  int parts;
  Layer<KIND, T> to;
};

// Workgroups of 8 waves that have half of a CU's LDS, or of 16 that have all of it.
template <int WAVES>
constexpr int kRoom = WAVES == 8 ? 64 << 10 : 130 << 10;

template <class T>
__host__ __device__ constexpr int steps_of(int n) { return (n * (int)sizeof(T) + kStepBytes - 1) / kStepBytes; }
__host__ __device__ constexpr int stage_pitch(int steps) { return steps * kStepBytes + 16; }  // 16 bytes on: rows of a fragment in different banks

// x's rows, zeros up to whole steps; rows of whole 16 bytes four chunks a lane at once.
template <class T>
__device__ __forceinline__ void stage_rows(char *stage, int steps, const T *x, int64_t ldx, int rows, int n, bool vec, int threads) {
  constexpr int N = 16 / sizeof(T);
  typedef T Chunk __attribute__((ext_vector_type(N)));
  const int units = steps * (kStepBytes / 16), total = rows * units, pitch = stage_pitch(steps);
  if (vec && n % N == 0) {
    for (int u0 = threadIdx.x; u0 < total; u0 += 4 * threads) {
      Chunk v[4];
      int at[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int u = min(u0 + i * threads, total - 1), r = u / units, c = u - r * units;
        at[i] = r * pitch + c * 16;
        v[i] = *(const Chunk *)(x + r * ldx + min(c * N, n - N));
        if (c * N >= n) v[i] = Chunk{};
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) *(Chunk *)(stage + at[i]) = v[i];
    }
  } else {
    for (int u = threadIdx.x; u < total; u += threads) {
      const int r = u / units, c = u - r * units;
      Chunk v = {};
#pragma unroll
      for (int i = 0; i < N; ++i)
        if (c * N + i < n) v[i] = x[r * ldx + c * N + i];
      *(Chunk *)(stage + r * pitch + c * 16) = v;
    }
  }
}

template <int KIND, class T, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 4) void k_few_rows(FewRows<KIND, T> p) {
  constexpr int kSteps = 2;  // a batch, while the next one is on its way
  __shared__ __attribute__((aligned(16))) char stage[kRoom<WAVES>];
  __shared__ f32x4 room[WAVES - 1][2][64];  // of all but the first wave, which is the first of its team
  const int lane = threadIdx.x & 63, wave = tile::uniform(threadIdx.x >> 6), i16 = lane & 15, j4 = lane >> 4;
  const int part = wave % p.parts, member = wave / p.parts, teams = WAVES / p.parts;
  const int wide = p.n * (int)sizeof(T), steps = steps_of<T>(p.n), per = (steps + p.parts - 1) / p.parts, s0 = part * per, s1 = min(s0 + per, steps);
  stage_rows(stage, steps, p.x, p.ldx, p.rows, p.n, p.vec_x, 64 * WAVES);
  __syncthreads();
  const char *from = stage + min(i16, p.rows - 1) * stage_pitch(steps) + j4 * 16;  // rows past the last repeat it; their sums go nowhere
  const int64_t hidden = p.to.hidden, turns = ceil_div(hidden, 16 * teams);
  for (int64_t turn = blockIdx.x; turn < turns; turn += gridDim.x) {
    const int64_t first = (turn * teams + member) * 16;
    const int there = (int)max((int64_t)0, min(hidden - first, (int64_t)16));
    const auto rows_of = [&](const char *w, int pitch) { return __builtin_amdgcn_make_buffer_rsrc((void *)(w + first * pitch), 0, there > 0 ? (there - 1) * pitch + wide : 0, 0x00027000); };
    const __amdgpu_buffer_rsrc_t rg = rows_of(p.wg, p.pitch_g), ru = rows_of(p.wu, p.pitch_u);
    struct Batch {
      i32x4 g[kSteps][2], u[kSteps][2];
    };
    // Steps from s on, zeros past s1. A row's last chunk may hold what follows the row: zeros take its place.
    const auto load = [&](Batch &to, int s) {
#pragma unroll
      for (int k = 0; k < kSteps; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = (s + k) * kStepBytes + h * 64 + j4 * 16;
          const bool in = s + k < s1 && at < wide;
          to.g[k][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(rg, in ? i16 * p.pitch_g + at : (int)tile::kOut, 0, 0));
          to.u[k][h] = __builtin_bit_cast(i32x4, __builtin_amdgcn_raw_buffer_load_b128(ru, in ? i16 * p.pitch_u + at : (int)tile::kOut, 0, 0));
        }
    };
    const auto clip = [&](i32x4 &v, int at) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = at + 4 * e < wide ? v[e] : 0;
    };
    f32x4 g = {0.0f, 0.0f, 0.0f, 0.0f}, u = g;
    if (s0 < s1) {
      Batch now, next;
      load(now, s0);
#pragma unroll 1
      for (int s = s0; s < s1; s += kSteps) {
        load(next, s + kSteps);
        if (wide % 16 && (s + kSteps) * kStepBytes > wide) {
#pragma unroll
          for (int k = 0; k < kSteps; ++k)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              clip(now.g[k][h], (s + k) * kStepBytes + h * 64 + j4 * 16);
              clip(now.u[k][h], (s + k) * kStepBytes + h * 64 + j4 * 16);
            }
        }
#pragma unroll
        for (int k = 0; k < kSteps; ++k)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const i32x4 x = *(const i32x4 *)(from + min(s + k, steps - 1) * kStepBytes + h * 64);  // (past the steps: products with zeros)
            g = tile::mfma<KIND>(now.g[k][h], x, g);
            u = tile::mfma<KIND>(now.u[k][h], x, u);
          }
        now = next;
      }
    }
    if (p.parts > 1) {
      if (part > 0) {
        room[wave - 1][0][lane] = g;
        room[wave - 1][1][lane] = u;
      }
      __syncthreads();
      if (part == 0)
        for (int w = 1; w < p.parts; ++w) {
          g += room[wave + w - 1][0][lane];
          u += room[wave + w - 1][1][lane];
        }
      __syncthreads();  // before the next turn's sums take the place
    }
    const int64_t c = first + 4 * j4;
    if (part == 0 && i16 < p.rows && c < hidden) {
      const int n = hidden - c < 4 ? (int)(hidden - c) : 4;
      if (p.to.gate) store4(p.to.gate + i16 * p.to.ldg + c, g, n, p.to.vec_g);
      if (p.to.up) store4(p.to.up + i16 * p.to.ldu + c, u, n, p.to.vec_u);
      if (p.to.h) store4(p.to.h + i16 * p.to.ldh + c, p.to.product(g, u), n, p.to.vec_h);
    }
  }
}

// ------------------------------------------------------------------------------------------------
// The gradient's dg and du

template <class T>
struct Slopes {
  const T *gate, *up, *dh;
  int64_t ldg, ldu, ldd;
  bool vec;  // the three's rows are aligned for 16 bytes
  int activation;
  int64_t rows, hidden, half;  // half: values of dg with its zeros
  char *out;
  int64_t pitch;  // bytes
};

template <class T, int N>
__device__ __forceinline__ void load_some(const T *row, int64_t c, int64_t n, bool vec, float (&v)[N]) {
  typedef T Chunk __attribute__((ext_vector_type(N)));
  if (vec && c + N <= n) {
    const Chunk x = *(const Chunk *)(row + c);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)x[i];
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = c + i < n ? (float)row[c + i] : 0.0f;
  }
}

// Where four values of a row's half go in the form of KIND.
template <int KIND>
__device__ __forceinline__ void store_slopes(char *row, int64_t c, const float *v) {
  const f32x4 x = {v[0], v[1], v[2], v[3]};
  if constexpr (KIND == KIND_THREE)
    store_three4(row, c, x);
  else if constexpr (KIND == KIND_F32)
    store4((float *)row + c, x, 4, true);
  else
    store4((__bf16 *)row + c, x, 4, true);
}

// 16 bytes of each input a lane. dg and du are rounded to bf16 once, between fp32 arithmetic and fp32 sums (bf16).
template <int KIND, class T>
__global__ __launch_bounds__(256) void k_slopes(Slopes<T> p) {
  constexpr int N = 16 / sizeof(T);
  for (int64_t t = blockIdx.y; t < p.rows; t += gridDim.y)
    for (int64_t c = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N; c < p.half; c += (int64_t)gridDim.x * 256 * N) {
      float g[N], u[N], d[N];
      load_some(p.gate + t * p.ldg, c, p.hidden, p.vec, g);
      load_some(p.up + t * p.ldu, c, p.hidden, p.vec, u);
      load_some(p.dh + t * p.ldd, c, p.hidden, p.vec, d);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const Activated a = activated<T, true>(p.activation, g[i]);
        g[i] = c + i < p.hidden ? d[i] * u[i] * a.slope : 0.0f;
        u[i] = c + i < p.hidden ? d[i] * a.value : 0.0f;
      }
      char *row = p.out + t * p.pitch;
      if constexpr (KIND == KIND_BF16) {
        typedef __bf16 Chunk __attribute__((ext_vector_type(N)));
        Chunk a, b;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          a[i] = (__bf16)g[i];
          b[i] = (__bf16)u[i];
        }
        *(Chunk *)((__bf16 *)row + c) = a;
        *(Chunk *)((__bf16 *)row + p.half + c) = b;
      } else {
        store_slopes<KIND>(row, c, g);
        store_slopes<KIND>(row, p.half + c, u);
      }
    }
}

// The two weights' gradients: rows [0, hidden) of the product are dwg's, those from `half` on dwu's.
template <class T>
struct TwoStores {
  using Value = T;
  T *gate, *up;  // either may be nullptr
  int64_t ldg, ldu, hidden, half;
  int64_t rows, cols;  // of the product: half + hidden
  bool vec;
  const float *factor = nullptr;
  __device__ __forceinline__ T *row(int64_t r) const {
    if (r < hidden) return gate ? gate + r * ldg : nullptr;
    return r >= half && r < rows && up ? up + (r - half) * ldu : nullptr;
  }
  template <class B>
  __device__ __forceinline__ void operator()(const B &block, int64_t row0, int64_t col0, int, bool) const {
#pragma unroll
    for (int i = 0; i < B::kTM; ++i) {
      T *to = row(row0 + 16 * i + (threadIdx.x & 15));
      store_row<T, B::kTN>(to, col0, cols, vec, to != nullptr, [&](int j) { return block.acc[i][j]; });
    }
  }
};

template <class T>
__global__ __launch_bounds__(256) void k_zero(T *out, int64_t ld, int64_t rows, int64_t cols) {
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
    for (int64_t c = threadIdx.x; c < cols; c += 256) out[r * ld + c] = (T)0.0f;
}

// ------------------------------------------------------------------------------------------------
// Host

struct Sizes {
  int64_t rows, hidden, features;
  int32_t dtype;
  bool plain() const { return rows <= kPlainRows || hidden <= kPlainHidden; }
  int kind() const { return dtype == SDNN_BF16 ? KIND_BF16 : plain() ? KIND_F32 : KIND_SPLIT; }
  bool small() const { return std::min(rows, hidden) <= kPlainSmall && rows * hidden <= kSmall / features; }
  int product_kind() const { return dtype == SDNN_BF16 ? KIND_BF16 : plain() || small() ? KIND_F32 : KIND_THREE; }  // the gradient's
  int bytes() const { return dtype_bytes(dtype); }
  // Bytes of a row of features written anew, as the layer and as the gradient take it.
  int64_t pitch(int kind) const {
    return kind == KIND_SPLIT ? ceil_div(features, 32) * 128 : kind == KIND_THREE ? ceil_div(features, 64) * tile::kGroup3 : ceil_div(features, 8) * 8 * bytes();
  }
  int64_t paired() const { return ceil_div(hidden, 16) * 32; }  // columns of the layer's product
  int64_t half() const { return ceil_div(hidden, 64) * 64; }    // values of dg in a row, whole slabs of any kind
  int64_t slopes_pitch() const { return product_kind() == KIND_THREE ? half() / 64 * 2 * tile::kGroup3 : half() * 2 * bytes(); }
  Plan layer() const { return plan(kind(), rows, paired(), features, rows * paired() <= kSplitValues && rows <= 65535 ? kMaxSplits : 1); }
  Plan dx() const { return product(rows, features, 2 * half()); }
  Plan dw() const { return product(half() + hidden, features, rows); }
  Plan product(int64_t m, int64_t n, int64_t k) const {
    const Plan p = plan(product_kind(), m, n, k, kMaxSplits);
    if (product_kind() != KIND_THREE) return p;
    const parts::Splits at_once = parts::plan(m, n, k, kMaxSplits);
    return at_once.us < p.us ? Plan{kShapes, at_once.splits, at_once.us} : p;
  }
  int64_t ld_slab() const { return ceil_div(features, 4) * 4; }
};

// x, wg and wu written anew. Room for all three is always taken: whether rows can be read in place is a matter of their
// addresses, which the workspace's size does not know.
struct Copies {
  char *x, *wg, *wu;
  int *ex, *eg, *eu;
  Copies(Carver &c, const Sizes &s, int kind) {
    x = c.take<char>((size_t)(s.rows * s.pitch(kind)));
    wg = c.take<char>((size_t)(s.hidden * s.pitch(kind)));
    wu = c.take<char>((size_t)(s.hidden * s.pitch(kind)));
    ex = c.take<int>(kind == KIND_SPLIT ? s.rows : 0);
    eg = c.take<int>(kind == KIND_SPLIT ? s.hidden : 0);
    eu = c.take<int>(kind == KIND_SPLIT ? s.hidden : 0);
  }
};

struct LayerSpace {
  Plan layer;
  Copies copies;
  float *slabs;
  LayerSpace(Carver &c, const Sizes &s) : layer(s.layer()), copies(c, s, s.kind()), slabs(c.take<float>(layer.splits > 1 ? (size_t)(layer.splits * s.rows * s.paired()) : 0)) {}
};

struct GradSpace {
  Plan dx, dw;
  Copies copies;
  char *slopes;
  float *dx_slabs, *dw_slabs;
  GradSpace(Carver &c, const Sizes &s) : dx(s.dx()), dw(s.dw()), copies(c, s, s.product_kind()) {
    slopes = c.take<char>((size_t)(s.rows * s.slopes_pitch()));
    dx_slabs = c.take<float>(dx.splits > 1 ? (size_t)(dx.splits * s.rows * s.ld_slab()) : 0);
    dw_slabs = c.take<float>(dw.splits > 1 ? (size_t)(dw.splits * (s.half() + s.hidden) * s.ld_slab()) : 0);
  }
};

template <class T>
struct Inputs {
  const T *x, *wg, *wu;
  int64_t ldx, ldg, ldu;
};

// x and the weights as operands of KIND, written anew where they have to be; nullptr space: not wanted.
struct Operands {
  Matrix x, w;  // w: two matrices
};
template <int KIND, class T>
sdnn_status operands(const Sizes &s, const Inputs<T> &in, const Copies &to, bool want_x, bool want_w, bool across, Operands &o, hipStream_t stream) {
  const T *data[3] = {in.x, in.wg, in.wu};
  const int64_t ld[3] = {in.ldx, in.ldg, in.ldu}, rows[3] = {s.rows, s.hidden, s.hidden};
  char *space[3] = {to.x, to.wg, to.wu};
  int *exponents[3] = {to.ex, to.eg, to.eu};
  const bool want[3] = {want_x, want_w, want_w};
  const char *base[3];
  int64_t pitch[3], extent = KIND == KIND_SPLIT ? s.pitch(KIND) : KIND == KIND_THREE ? ceil_div(s.features, 8) * 16 : s.features * (int64_t)sizeof(T);
  constexpr bool kParts = KIND == KIND_SPLIT || KIND == KIND_THREE;
  // each is read in place or written anew; a row written anew is at least as long as what is read of it
  bool in_place[3];
  for (int i = 0; i < 3; ++i) in_place[i] = !kParts && usable_in_place(data[i], ld[i], s.features, sizeof(T));
  if (s.features * sizeof(T) % 4) extent = s.pitch(KIND);  // no row is usable in place then
  Sources src{};
  src.cols = s.features;
  int64_t all = 0;
  for (int i = 0; i < 3; ++i) {
    const bool write = want[i] && !in_place[i];
    src.of[i] = {data[i], ld[i], write ? rows[i] : 0, space[i], exponents[i], aligned16(data[i], ld[i], sizeof(T))};
    all += src.of[i].rows;
    base[i] = in_place[i] ? (const char *)data[i] : space[i];
    pitch[i] = in_place[i] ? ld[i] * (int64_t)sizeof(T) : s.pitch(KIND);
  }
  if (all > 0) {
    const dim3 grid((unsigned)std::min<int64_t>(all, 4096));
    if constexpr (KIND == KIND_SPLIT)
      hipLaunchKernelGGL(k_two_parts, grid, dim3(256), 0, stream, src, all);
    else if constexpr (KIND == KIND_THREE)
      hipLaunchKernelGGL(k_three_parts, grid, dim3(256), 0, stream, src, all);
    else
      hipLaunchKernelGGL((k_aligned<T>), grid, dim3(256), 0, stream, src, all);
    const sdnn_status st = launched("rows");
    if (st != SDNN_OK) return st;
  }
  o.x = {base[0], pitch[0], s.rows, extent, 0};
  o.w = {base[1], pitch[1], s.hidden, extent, 0};
  o.w.second = base[2];
  o.w.pitch_second = pitch[2];
  if (across) o.w.units = (int)(s.half() / tile::Geometry<KIND>::kPerSlab);
  return SDNN_OK;
}

template <class T>
struct Kept {
  T *gate, *up;
  int64_t ldg, ldu;
};

// Few rows whose weights are read where they are. us, here and in tiles: bf16 1 x 1024 to 4096 8.3 / 10.1, 1 x 4096 to 16384 50 / 64,
// 16 x 4096 to 16384 55 / 68, 8 x 16384 to 4096 62 / 63; fp32 1 x 4096 to 8192 58 / 70, 16 x 1000 to 100 9.8 / 10.1.
template <class T>
bool few_rows(const Sizes &s, const Inputs<T> &in) {
  return s.rows <= 16 && s.rows * (int64_t)stage_pitch(steps_of<T>((int)s.features)) <= kRoom<16> && usable_in_place(in.wg, in.ldg, s.features, sizeof(T)) &&
         usable_in_place(in.wu, in.ldu, s.features, sizeof(T));
}

template <int KIND, class T, int WAVES>
sdnn_status launch_few(FewRows<KIND, T> p, hipStream_t stream) {
  const int64_t tiles = ceil_div(p.to.hidden, 16);
  // as many waves on an output's k as it takes to give every CU 16
  p.parts = 1;
  while (p.parts < WAVES && tiles * p.parts < 16 * kCus && p.parts * 2 <= steps_of<T>(p.n)) p.parts *= 2;
  const dim3 grid((unsigned)std::min<int64_t>(ceil_div(tiles, WAVES / p.parts), 16 / WAVES * kCus));
  hipLaunchKernelGGL((k_few_rows<KIND, T, WAVES>), grid, dim3(64 * WAVES), 0, stream, p);
  return launched("gated layer");
}

template <int KIND, class T>
sdnn_status layer_of(const Sizes &s, const Inputs<T> &in, int activation, T *h, int64_t ldh, const Kept<T> &kept, Carver &carver, hipStream_t stream) {
  const LayerSpace sp(carver, s);
  const Layer<KIND, T> e{sp.copies.ex, sp.copies.eg, sp.copies.eu, activation, s.rows, s.hidden, h, kept.gate, kept.up, ldh, kept.ldg, kept.ldu,
                         vector_rows(h, ldh), vector_rows(kept.gate, kept.ldg), vector_rows(kept.up, kept.ldu)};
  if constexpr (KIND != KIND_SPLIT) {
    if (few_rows(s, in)) {
      const FewRows<KIND, T> p{in.x, in.ldx, aligned16(in.x, in.ldx, sizeof(T)), (int)s.rows, (int)s.features, (const char *)in.wg, (const char *)in.wu, (int)(in.ldg * (int64_t)sizeof(T)),
                               (int)(in.ldu * (int64_t)sizeof(T)), 1, e};
      return s.rows * stage_pitch(steps_of<T>((int)s.features)) <= kRoom<8> ? launch_few<KIND, T, 8>(p, stream) : launch_few<KIND, T, 16>(p, stream);
    }
  }
  Operands o;
  sdnn_status st = operands<KIND>(s, in, sp.copies, true, true, false, o, stream);
  if (st != SDNN_OK) return st;
  if (sp.layer.splits == 1) return run_shape<KIND, false, false, true>(sp.layer, o.x, o.w, s.rows, s.paired(), s.features, e, stream, "gated layer");
  const int64_t ld = s.paired();
  st = run_shape<KIND, false, false, true>(sp.layer, o.x, o.w, s.rows, ld, s.features, Accumulate{sp.slabs, ld, s.rows, ld, false}, stream, "gated layer");
  if (st != SDNN_OK) return st;
  hipLaunchKernelGGL((k_layer_slabs<KIND, T>), dim3((unsigned)std::min<int64_t>(ceil_div(s.hidden, 1024), 256), (unsigned)s.rows), dim3(256), 0, stream, sp.slabs, sp.layer.splits, ld, e);
  return launched("gated layer");
}

// Workgroups along a row of `items` lanes, and down the rows.
dim3 grid_of(int64_t rows, int64_t items) {
  const int64_t x = ceil_div(items, 256);
  return dim3((unsigned)x, (unsigned)std::max<int64_t>(1, std::min<int64_t>({rows, 65535, ceil_div(kCus * 32, x)})));
}

template <class T>
struct Gradients {
  T *dx, *dwg, *dwu;
  int64_t lddx, lddg, lddu;
};

// A product of the gradient by its plan: kShapes stands for blocks whose parts lie in LDS at once.
template <int KIND, bool AA, bool AB, bool TWO, class E, class Tail = NoTail>
sdnn_status product(const Plan &p, const Matrix &a, const Matrix &b, int64_t rows, int64_t cols, int64_t k, const E &e, hipStream_t stream, const char *what, const Tail &tail = {}) {
  if constexpr (KIND == KIND_THREE)
    if (p.shape == kShapes) return parts::launch<AA, AB, TWO>(a, b, rows, cols, k, p.splits, e, stream, what, tail);
  return run_shape<KIND, AA, AB, TWO>(p, a, b, rows, cols, k, e, stream, what, false, 1, tail);
}

template <int kProduct, class T>
sdnn_status grad_of(const Sizes &s, const Inputs<T> &in, int activation, const Kept<T> &kept, const T *dh, int64_t lddh, const Gradients<T> &to, Carver &carver, hipStream_t stream) {
  const GradSpace sp(carver, s);
  const bool weights = to.dwg || to.dwu;
  const Slopes<T> p{kept.gate, kept.up, dh, kept.ldg, kept.ldu, lddh, vector_rows(kept.gate, kept.ldg) && vector_rows(kept.up, kept.ldu) && vector_rows(dh, lddh), activation,
                    s.rows, s.hidden, s.half(), sp.slopes, s.slopes_pitch()};
  hipLaunchKernelGGL((k_slopes<kProduct, T>), grid_of(s.rows, ceil_div(s.half(), 16 / (int)sizeof(T))), dim3(256), 0, stream, p);
  sdnn_status st = launched("gated gradient");
  if (st != SDNN_OK) return st;
  Operands o;
  st = operands<kProduct>(s, in, sp.copies, weights, to.dx != nullptr, true, o, stream);
  if (st != SDNN_OK) return st;
  const int64_t per_value = kProduct == KIND_THREE ? 2 : (int64_t)sizeof(T), ld = s.ld_slab();
  const Matrix d{sp.slopes, s.slopes_pitch(), s.rows, 2 * s.half() * per_value, 0};
  // dx's split sums are joined by the weights' launch where there is one
  const Store<T> ex{to.dx, to.lddx, s.rows, s.features, vector_rows(to.dx, to.lddx)};
  SumTail<Store<T>> tail{nullptr, 0, 0, 1, ld, ex};
  if (to.dx) {
    const char *what = "gated gradient of the rows";
    if (sp.dx.splits == 1) {
      st = product<kProduct, false, true, true>(sp.dx, d, o.w, s.rows, s.features, 2 * s.half(), ex, stream, what);
    } else {
      st = product<kProduct, false, true, true>(sp.dx, d, o.w, s.rows, s.features, 2 * s.half(), Accumulate{sp.dx_slabs, ld, s.rows, s.features, false}, stream, what);
      if (weights)
        tail = sum_tail(sp.dx_slabs, sp.dx.splits, ld, ex);
      else if (st == SDNN_OK)
        st = sum_slabs(sp.dx_slabs, sp.dx.splits, ld, ex, stream, what);
    }
    if (st != SDNN_OK) return st;
  }
  if (weights) {
    const char *what = "gated gradient of the weights";
    const int64_t rows = s.half() + s.hidden;
    const TwoStores<T> e{to.dwg, to.dwu, to.lddg, to.lddu, s.hidden, s.half(), rows, s.features,
                         (!to.dwg || vector_rows(to.dwg, to.lddg)) && (!to.dwu || vector_rows(to.dwu, to.lddu))};
    if (sp.dw.splits == 1) {
      st = product<kProduct, true, true, false>(sp.dw, d, o.x, rows, s.features, s.rows, e, stream, what, tail);
    } else {
      st = product<kProduct, true, true, false>(sp.dw, d, o.x, rows, s.features, s.rows, Accumulate{sp.dw_slabs, ld, rows, s.features, false}, stream, what, tail);
      if (st == SDNN_OK) st = sum_slabs(sp.dw_slabs, sp.dw.splits, ld, e, stream, what);
    }
  }
  return st;
}

sdnn_status check_sizes(int64_t n_rows, int64_t n_hidden, int64_t n_features, int32_t dtype) {
  if (n_rows < 0 || n_rows > kMaxRows) return fail(SDNN_EINVAL, "n_rows %lld is outside [0, %lld]", (long long)n_rows, (long long)kMaxRows);
  if (n_hidden < 1 || n_hidden > kMaxHidden) return fail(SDNN_EINVAL, "n_hidden %lld is outside [1, %lld]", (long long)n_hidden, (long long)kMaxHidden);
  if (n_features < 1 || n_features > kMaxFeatures) return fail(SDNN_EINVAL, "n_features %lld is outside [1, %lld]", (long long)n_features, (long long)kMaxFeatures);
  if (!good_dtype(dtype)) return fail(SDNN_EINVAL, "dtype %d is neither SDNN_FP32 nor SDNN_BF16", dtype);
  return SDNN_OK;
}

sdnn_status check_activation(int32_t activation) {
  if (activation < SDNN_SILU || activation > SDNN_RELU) return fail(SDNN_EINVAL, "activation %d is none of SDNN_SILU, SDNN_GELU and SDNN_RELU", activation);
  return SDNN_OK;
}

enum Gradient { kLayerOnly = 0, kFromKept = 1, kAgain = 2 };

// The parts of a gradient call's workspace: g and u where they are computed again (and what the layer needs for it), then
// the gradient's own over the same room.
template <class T>
Kept<T> again_space(Carver &c, const Sizes &s) {
  const int64_t ld = ceil_div(s.hidden, 8) * 8;
  T *gate = c.take<T>((size_t)(s.rows * ld)), *up = c.take<T>((size_t)(s.rows * ld));
  return {gate, up, ld, ld};
}

size_t workspace_of(const Sizes &s, int gradient) {
  Carver layer{nullptr};
  if (gradient == kAgain) {
    if (s.dtype == SDNN_BF16)
      again_space<__bf16>(layer, s);
    else
      again_space<float>(layer, s);
  }
  Carver grad = layer;
  LayerSpace a(layer, s);
  if (gradient == kLayerOnly) return layer.used;
  GradSpace b(grad, s);
  return std::max(layer.used, grad.used);
}

template <class T>
sdnn_status layer_call(const Sizes &s, const Inputs<T> &in, int activation, T *h, int64_t ldh, const Kept<T> &kept, Carver &c, hipStream_t stream) {
  if constexpr (sizeof(T) == 2)
    return layer_of<KIND_BF16>(s, in, activation, h, ldh, kept, c, stream);
  else
    return s.kind() == KIND_F32 ? layer_of<KIND_F32>(s, in, activation, h, ldh, kept, c, stream) : layer_of<KIND_SPLIT>(s, in, activation, h, ldh, kept, c, stream);
}

template <class T>
sdnn_status grad_call(const Sizes &s, const Inputs<T> &in, int activation, Kept<T> kept, const T *dh, int64_t lddh, const Gradients<T> &to, Carver c, hipStream_t stream) {
  if (!kept.gate) {
    kept = again_space<T>(c, s);
    Carver over = c;
    const sdnn_status st = layer_call<T>(s, in, activation, nullptr, 0, kept, over, stream);
    if (st != SDNN_OK) return st;
  }
  if constexpr (sizeof(T) == 2)
    return grad_of<KIND_BF16>(s, in, activation, kept, dh, lddh, to, c, stream);
  else
    return s.product_kind() == KIND_F32 ? grad_of<KIND_F32>(s, in, activation, kept, dh, lddh, to, c, stream) : grad_of<KIND_THREE>(s, in, activation, kept, dh, lddh, to, c, stream);
}

template <class T>
void zero(void *p, int64_t ld, const Sizes &s, hipStream_t stream) {
  if (p) hipLaunchKernelGGL((k_zero<T>), dim3(row_grid(s.hidden)), dim3(256), 0, stream, (T *)p, ld, s.hidden, s.features);
}

}  // namespace

extern "C" {

size_t sdnn_gated_workspace_bytes(int64_t n_rows, int64_t n_hidden, int64_t n_features, int32_t dtype, int32_t gradient) {
  if (check_sizes(n_rows, n_hidden, n_features, dtype) != SDNN_OK || gradient < kLayerOnly || gradient > kAgain) return 0;
  return workspace_of({n_rows, n_hidden, n_features, dtype}, gradient);
}

sdnn_status sdnn_gated(const void *x, int64_t ldx, const void *w_gate, int64_t ldw_gate, const void *w_up, int64_t ldw_up, int32_t dtype, int32_t activation, int64_t n_rows, int64_t n_hidden,
                       int64_t n_features, void *h, int64_t ldh, void *gate, int64_t ldgate, void *up, int64_t ldup, void *workspace, size_t workspace_bytes, void *hip_stream) {
  sdnn_status st = check_sizes(n_rows, n_hidden, n_features, dtype);
  if (st == SDNN_OK) st = check_activation(activation);
  if (st != SDNN_OK || n_rows == 0) return st;
  if ((st = check_matrix("x", x, ldx, n_features, dtype)) != SDNN_OK) return st;
  if ((st = check_matrix("w_gate", w_gate, ldw_gate, n_features, dtype)) != SDNN_OK) return st;
  if ((st = check_matrix("w_up", w_up, ldw_up, n_features, dtype)) != SDNN_OK) return st;
  if ((st = check_matrix("h", h, ldh, n_hidden, dtype)) != SDNN_OK) return st;
  if (gate && (st = check_matrix("gate", gate, ldgate, n_hidden, dtype)) != SDNN_OK) return st;
  if (up && (st = check_matrix("up", up, ldup, n_hidden, dtype)) != SDNN_OK) return st;
  const Sizes s{n_rows, n_hidden, n_features, dtype};
  if ((st = check_workspace(workspace, workspace_bytes, workspace_of(s, kLayerOnly))) != SDNN_OK) return st;
  const hipStream_t stream = (hipStream_t)hip_stream;
  const auto call = [&](auto value) {
    using T = decltype(value);
    Carver c{(char *)workspace};
    return layer_call<T>(s, {(const T *)x, (const T *)w_gate, (const T *)w_up, ldx, ldw_gate, ldw_up}, activation, (T *)h, ldh, {(T *)gate, (T *)up, ldgate, ldup}, c, stream);
  };
  return dtype == SDNN_BF16 ? call((__bf16)0.0f) : call(0.0f);
}

sdnn_status sdnn_gated_grad(const void *x, int64_t ldx, const void *w_gate, int64_t ldw_gate, const void *w_up, int64_t ldw_up, int32_t dtype, int32_t activation, const void *gate, int64_t ldgate,
                            const void *up, int64_t ldup, const void *dh, int64_t lddh, int64_t n_rows, int64_t n_hidden, int64_t n_features, void *dx, int64_t lddx, void *dw_gate, int64_t lddw_gate,
                            void *dw_up, int64_t lddw_up, void *workspace, size_t workspace_bytes, void *hip_stream) {
  sdnn_status st = check_sizes(n_rows, n_hidden, n_features, dtype);
  if (st == SDNN_OK) st = check_activation(activation);
  if (st != SDNN_OK) return st;
  if (n_rows > 0) {
    if ((st = check_matrix("x", x, ldx, n_features, dtype)) != SDNN_OK) return st;
    if ((st = check_matrix("w_gate", w_gate, ldw_gate, n_features, dtype)) != SDNN_OK) return st;
    if ((st = check_matrix("w_up", w_up, ldw_up, n_features, dtype)) != SDNN_OK) return st;
    if ((st = check_matrix("dh", dh, lddh, n_hidden, dtype)) != SDNN_OK) return st;
    if (!gate != !up) return fail(SDNN_EINVAL, "gate and up are kept together or not at all");
    if (gate && (st = check_matrix("gate", gate, ldgate, n_hidden, dtype)) != SDNN_OK) return st;
    if (up && (st = check_matrix("up", up, ldup, n_hidden, dtype)) != SDNN_OK) return st;
    if (dx && (st = check_matrix("dx", dx, lddx, n_features, dtype)) != SDNN_OK) return st;
  }
  if (dw_gate && (st = check_matrix("dw_gate", dw_gate, lddw_gate, n_features, dtype)) != SDNN_OK) return st;
  if (dw_up && (st = check_matrix("dw_up", dw_up, lddw_up, n_features, dtype)) != SDNN_OK) return st;
  if ((!dx || n_rows == 0) && !dw_gate && !dw_up) return SDNN_OK;
  const Sizes s{n_rows, n_hidden, n_features, dtype};
  const hipStream_t stream = (hipStream_t)hip_stream;
  if (n_rows == 0) {
    for (const auto &[p, ld] : {std::pair<void *, int64_t>{dw_gate, lddw_gate}, std::pair<void *, int64_t>{dw_up, lddw_up}}) dtype == SDNN_BF16 ? zero<__bf16>(p, ld, s, stream) : zero<float>(p, ld, s, stream);
    return launched("gated gradient");
  }
  if ((st = check_workspace(workspace, workspace_bytes, workspace_of(s, gate ? kFromKept : kAgain))) != SDNN_OK) return st;
  const auto call = [&](auto value) {
    using T = decltype(value);
    return grad_call<T>(s, {(const T *)x, (const T *)w_gate, (const T *)w_up, ldx, ldw_gate, ldw_up}, activation, {(T *)gate, (T *)up, ldgate, ldup}, (const T *)dh, lddh,
                        {(T *)dx, (T *)dw_gate, (T *)dw_up, lddx, lddw_gate, lddw_up}, Carver{(char *)workspace}, stream);
  };
  return dtype == SDNN_BF16 ? call((__bf16)0.0f) : call(0.0f);
}

}  // extern "C"
