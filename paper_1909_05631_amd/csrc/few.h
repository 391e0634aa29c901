// The readout of few rows or of few classes, in fp32 arithmetic without matrix tiles: the few (the "held" rows of x or of
// w, at most 4) stay in registers, spread over a workgroup's columns, while the rows of the other matrix
// stream past, each read once:
//
//   l_hs = held_h . stream_s           per lane over its columns, then across the workgroup
//   loss:     rows held: a running maximum and sum of each row over the classes that pass; classes held: a row's
//             whole softmax as it passes
//   gradient: G_hs from l_hs and the given lse;  d stream_s = sum_h G_hs held_h  is written,
//             d held_h += G_hs stream_s  stays in registers, one slab per workgroup at the end
//
// Bound by memory where rows are long (the streamed matrix once, its gradient once: 65536 x 1024 fp32 against one row 45 us,
// 6.0 TB/s), by the sums across lanes where they are short. A sum across 64 lanes of N values takes N + log2(64 / N)
// shuffles: each step a lane hands on the half of the values that its neighbour keeps.
#ifndef SDNN_FEW_H
#define SDNN_FEW_H

#include "dense.h"

#include <type_traits>

namespace few {

using namespace dense;

constexpr int kThreads = 256, kWaves = 4, kColumns = 4 * kThreads;  // columns of one step across the workgroup

template <class T>
struct Few {
  const T *held, *stream;
  int64_t ld_held, ld_stream;
  int held_rows, features;
  int64_t stream_rows;
  bool vec_held, vec_stream;  // rows aligned for four values, features a multiple of four
  const int64_t *labels;
  int64_t classes;
  // loss
  float *loss, *lse;      // classes held
  float2 *parts;          // rows held: [row][parts of the launch]
  float *picked;
  // gradient
  const float *known_lse, *weights, *mean;  // weights == nullptr: the mean over the counted rows (rows held: counted here)
  T *d_stream;            // nullptr: not wanted
  int64_t ld_d;
  bool vec_d;
  float *slabs;           // nullptr: not wanted; [workgroup][held row][ld_slab]
  int64_t ld_slab;
};

template <class T>
__device__ __forceinline__ f32x4 load4(const T *row, int col, int n, bool vec) {
  typedef T T4 __attribute__((ext_vector_type(4)));
  f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if (vec && col + 4 <= n) {
    v = __builtin_convertvector(*(const T4 *)(row + col), f32x4);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (col + i < n) v[i] = (float)row[col + i];
  }
  return v;
}

// A row as a buffer: reads past its end, and all reads of a row that is left out, are zeros without a branch, so
// that a thread's loads are all on their way at once.
template <class T>
struct RowBuffer {
  __amdgpu_buffer_rsrc_t r;
  __device__ __forceinline__ RowBuffer(const T *row, int n, bool live) : r(__builtin_amdgcn_make_buffer_rsrc((void *)row, 0, live ? n * (int)sizeof(T) : 0, 0x00027000)) {}
  // VEC: the row is aligned for four values and n is a multiple of four
  template <bool VEC>
  __device__ __forceinline__ f32x4 load(int col) const {
    typedef T T4 __attribute__((ext_vector_type(4)));
    const int at = col * (int)sizeof(T);
    if constexpr (VEC && sizeof(T) == 4) {
      return __builtin_bit_cast(f32x4, __builtin_amdgcn_raw_buffer_load_b128(r, at, 0, 0));
    } else if constexpr (VEC) {
      return __builtin_convertvector(__builtin_bit_cast(T4, __builtin_amdgcn_raw_buffer_load_b64(r, at, 0, 0)), f32x4);
    } else {
      f32x4 v;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if constexpr (sizeof(T) == 4)
          v[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, at + 4 * i, 0, 0));
        else
          v[i] = (float)__builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b16(r, at + 2 * i, 0, 0));
      return v;
    }
  }
};

__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896340736f); }

// Sums of v over the wave's lanes; lane i < N returns the sum of v[place(i)].
template <int N>
__device__ __forceinline__ float sum_lanes(float (&v)[N]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int n = N, m = 1; n > 1; n /= 2, m *= 2) {
    const bool upper = lane & m;
#pragma unroll
    for (int i = 0; i < n / 2; ++i) {
      const float keep = upper ? v[n / 2 + i] : v[i], pass = upper ? v[i] : v[n / 2 + i];
      v[i] = keep + __shfl_xor(pass, m);
    }
  }
  float s = v[0];
#pragma unroll
  for (int m = N; m < 64; m *= 2) s += __shfl_xor(s, m);
  return s;
}
template <int N>
__device__ __forceinline__ int place(int lane) {
  int p = 0;
#pragma unroll
  for (int n = N / 2, b = 0; n >= 1; n /= 2, ++b) p += (lane >> b & 1) * n;
  return p;
}

// HELD rows of at most kColumns * STEPS columns; BATCH streamed rows at a time.
template <class T, int HELD, int STEPS, int BATCH, bool ROWS_HELD, bool GRADIENT>
__global__ __launch_bounds__(kThreads) void k_few(Few<T> p) {
  constexpr int N = HELD * BATCH;  // sums of a batch: [held][streamed]
  __shared__ float part[2][kWaves][N];
  __shared__ __attribute__((aligned(16))) float shared_g[2][N];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  f32x4 held[HELD][STEPS], d_held[GRADIENT ? HELD : 1][GRADIENT ? STEPS : 1];
  int labelled = 0;
  bool takes[HELD];  // a row without a label is zeros in the gradient, whatever it holds
#pragma unroll
  for (int h = 0; h < HELD; ++h) {
    const bool there = h < p.held_rows, live = ROWS_HELD && there && (uint64_t)p.labels[h] < (uint64_t)p.classes;
    labelled += live;
    takes[h] = there && (!ROWS_HELD || !GRADIENT || live);
  }
  const auto load_held = [&](auto vec) {
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
      const RowBuffer<T> row(p.held + h * p.ld_held, p.features, takes[h]);
#pragma unroll
      for (int c = 0; c < STEPS; ++c) held[h][c] = row.template load<vec()>((c * kThreads + tid) * 4);
    }
  };
  if (p.vec_held)
    load_held(std::true_type{});
  else
    load_held(std::false_type{});
  if constexpr (GRADIENT) {
#pragma unroll
    for (int h = 0; h < HELD; ++h)
#pragma unroll
      for (int c = 0; c < STEPS; ++c) d_held[h][c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // this thread's sum of a batch
  const int mine = tid < N ? tid : 0, my_h = mine / BATCH, my_s = mine % BATCH;
  const bool my_held = tid < N && my_h < p.held_rows;
  const int64_t my_label = ROWS_HELD && my_held ? p.labels[my_h] : -1;
  float my_weight = 0.0f, my_lse = 0.0f;
  if (GRADIENT && ROWS_HELD && my_held && (uint64_t)my_label < (uint64_t)p.classes) {
    my_lse = p.known_lse[my_h];
    my_weight = p.weights ? p.weights[my_h] : 1.0f / labelled;
  }
  const bool my_live = (uint64_t)my_label < (uint64_t)p.classes;
  const float mean = GRADIENT && !ROWS_HELD && !p.weights ? *p.mean : 0.0f;
  float top = -__builtin_inff(), sum = 0.0f;  // loss, rows held

  const int64_t stride = (int64_t)gridDim.x * BATCH;
  f32x4 v[BATCH][STEPS];
  const auto load_rows = [&](int64_t s0, auto vec) {
#pragma unroll
    for (int b = 0; b < BATCH; ++b) {
      const int64_t s = s0 + b;
      const bool live = s < p.stream_rows && (ROWS_HELD || !GRADIENT || (uint64_t)p.labels[s] < (uint64_t)p.classes);
      const RowBuffer<T> row(p.stream + s * p.ld_stream, p.features, live);
#pragma unroll
      for (int c = 0; c < STEPS; ++c) v[b][c] = row.template load<vec()>((c * kThreads + tid) * 4);
    }
  };
  const auto load = [&](int64_t s0) {
    if (p.vec_stream)
      load_rows(s0, std::true_type{});
    else
      load_rows(s0, std::false_type{});
  };
  int64_t s0 = (int64_t)blockIdx.x * BATCH;
  load(s0);
  for (int turn = 0; s0 < p.stream_rows; s0 += stride, turn ^= 1) {
    float dots[N];
#pragma unroll
    for (int h = 0; h < HELD; ++h)
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        float d = 0.0f;
#pragma unroll
        for (int c = 0; c < STEPS; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i) d = fmaf(held[h][c][i], v[b][c][i], d);
        dots[h * BATCH + b] = d;
      }
    f32x4 now[GRADIENT ? BATCH : 1][GRADIENT ? STEPS : 1];
    if constexpr (GRADIENT) {
#pragma unroll
      for (int b = 0; b < BATCH; ++b)
#pragma unroll
        for (int c = 0; c < STEPS; ++c) now[b][c] = v[b][c];
    }
    if constexpr (STEPS < 16 || !GRADIENT) load(s0 + stride);  // the next batch's rows are on their way while this one's sums meet
    const float s = sum_lanes(dots);
    if (lane < N) part[turn][wave][place<N>(lane)] = s;
    __syncthreads();
    float l = 0.0f;
    if (tid < N) {
#pragma unroll
      for (int w = 0; w < kWaves; ++w) l += part[turn][w][tid];
    }
    const int64_t s_mine = s0 + my_s;
    const bool in = my_held && s_mine < p.stream_rows;
    if constexpr (!GRADIENT && ROWS_HELD) {
      if (in) {
        if (s_mine == my_label) p.picked[my_h] = l;
        const float n = fmaxf(top, l);
        sum = (top == -__builtin_inff() ? sum : sum * exp_of(top - n)) + (l == -__builtin_inff() ? 0.0f : exp_of(l - n));
        top = n;
      }
    } else if constexpr (!GRADIENT) {
      if (tid < N) shared_g[turn][tid] = l;
      __syncthreads();
      if (tid < BATCH && s0 + tid < p.stream_rows) {
        float m = -__builtin_inff(), e = 0.0f;
        for (int h = 0; h < p.held_rows; ++h) m = fmaxf(m, shared_g[turn][h * BATCH + tid]);
        for (int h = 0; h < p.held_rows; ++h) {
          const float x = shared_g[turn][h * BATCH + tid];
          e += x == -__builtin_inff() ? 0.0f : exp_of(x - m);
        }
        const float z = m + logf(e);
        const int64_t y = p.labels[s0 + tid];
        if (p.lse) p.lse[s0 + tid] = z;
        p.loss[s0 + tid] = (uint64_t)y < (uint64_t)p.classes ? z - shared_g[turn][y * BATCH + tid] : 0.0f;
      }
    } else {
      if (tid < N) {
        float g = 0.0f;
        if (ROWS_HELD) {
          if (in && my_live) g = my_weight * (exp_of(l - my_lse) - (s_mine == my_label ? 1.0f : 0.0f));
        } else if (in) {
          const int64_t y = p.labels[s_mine];
          if ((uint64_t)y < (uint64_t)p.classes) g = (p.weights ? p.weights[s_mine] : mean) * (exp_of(l - p.known_lse[s_mine]) - (my_h == y ? 1.0f : 0.0f));
        }
        shared_g[turn][tid] = g;
      }
      __syncthreads();
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        f32x4 d[STEPS];
#pragma unroll
        for (int c = 0; c < STEPS; ++c) d[c] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        // a streamed row without a label has a gradient of zeros, whatever the held rows hold
        const bool live = s0 + b < p.stream_rows && (ROWS_HELD || (uint64_t)p.labels[s0 + b] < (uint64_t)p.classes);
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
          const float g = shared_g[turn][h * BATCH + b];
#pragma unroll
          for (int c = 0; c < STEPS; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              d[c][i] = fmaf(g, held[h][c][i], d[c][i]);
              d_held[h][c][i] = fmaf(g, now[b][c][i], d_held[h][c][i]);
            }
        }
        if (p.d_stream && s0 + b < p.stream_rows)
#pragma unroll
          for (int c = 0; c < STEPS; ++c) {
            const int col = (c * kThreads + tid) * 4;
            if (col < p.features) store4(p.d_stream + (s0 + b) * p.ld_d + col, live ? d[c] : f32x4{0.0f, 0.0f, 0.0f, 0.0f}, min(p.features - col, 4), p.vec_d);
          }
      }
      if constexpr (STEPS >= 16) load(s0 + stride);
    }
  }
  if constexpr (!GRADIENT && ROWS_HELD) {
    if (my_held) p.parts[my_h * ((int64_t)gridDim.x * BATCH) + blockIdx.x * BATCH + my_s] = float2{top, sum};
  }
  if constexpr (GRADIENT) {
    if (p.slabs)
#pragma unroll
      for (int h = 0; h < HELD; ++h)
#pragma unroll
        for (int c = 0; c < STEPS; ++c) {
          const int64_t col = (c * kThreads + tid) * 4;
          if (h < p.held_rows && col < p.ld_slab) *(f32x4 *)(p.slabs + ((int64_t)blockIdx.x * p.held_rows + h) * p.ld_slab + col) = d_held[h][c];
        }
  }
}

// The held rows and columns that registers take, and how many streamed rows go at a time: up to 4 rows in fp32, one in
// bf16, where all of the few go at once (two bf16 rows are far ahead in tiles). Past that it is a matter of two costs.
// A streamed row costs its sum across the workgroup, about 2 ns for four held rows, whatever its length; the tiles
// cost launches (us for the loss / the gradient, here and in tiles):
//   few streamed rows, where launches count: 4 x 2048 x 1024 fp32 13/18 and 19/28, 4 x 8192 x 1024 22/47 and 25/46,
//     one row of bf16 8192 x 1024 12/18 and 12/29, 1000 x 16384 13/31 and 31/41 (but 4096 x 16384 33/132 and 38/98);
//   many rows: only long ones are worth their sums. Four held, fp32: 200000 x 100 381/882 and 46/139, 30000 x 1500
//     52/173 and 41/139, 30000 x 2048 53/183 and 49/196, 32768 x 4096 95/261 and 123/428. One, fp32: 100000 x 256
//     49/117 and 40/109, 100000 x 512 50/143 and 62/174, 65536 x 1024 45/127 and 56/230. One, bf16: 200000 x 100 121/315
//     and 24/89, 30000 x 2048 37/88 and 25/91, 32768 x 4096 42/140 and 47/222, 16384 x 8192 94/328 and 85/235.
enum Fit { kNone, kOneShort, kOneMiddle, kOneLong, kFourShort, kFourMiddle };
inline Fit fit_of(int64_t held, int64_t streamed, int64_t features, int32_t dtype) {
  const bool fp32 = dtype == SDNN_FP32;
  if (held > (fp32 ? 4 : 1) || features > (held > 1 ? 4 : 16) * kColumns) return kNone;
  const bool long_bf16 = !fp32 && features > 4 * kColumns;
  if (streamed > (long_bf16 ? 1024 : 8192) && (long_bf16 || (fp32 ? features < (held > 1 ? 2048 : 512) : features <= 2048))) return kNone;
  if (held > 1) return features <= kColumns ? kFourShort : kFourMiddle;
  return features <= kColumns ? kOneShort : features <= 4 * kColumns ? kOneMiddle : kOneLong;
}
inline int batch_of(Fit f) { return f == kOneShort ? 8 : f == kFourShort ? 4 : f == kOneLong ? 1 : 2; }
// Workgroups: two a CU (each has 16 KB or more of rows on its way), one where each leaves a slab.
inline unsigned grid_of(Fit f, int64_t stream_rows, bool gradient) {
  return (unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(stream_rows, batch_of(f)), gradient ? kCus : 2 * kCus));
}

template <bool ROWS_HELD, bool GRADIENT, class T>
sdnn_status launch(Fit fit, const Few<T> &p, hipStream_t stream, const char *what) {
  const dim3 grid(grid_of(fit, p.stream_rows, GRADIENT)), threads(kThreads);
  switch (fit) {
    case kOneShort: hipLaunchKernelGGL((k_few<T, 1, 1, 8, ROWS_HELD, GRADIENT>), grid, threads, 0, stream, p); break;
    case kOneMiddle: hipLaunchKernelGGL((k_few<T, 1, 4, 2, ROWS_HELD, GRADIENT>), grid, threads, 0, stream, p); break;
    case kOneLong: hipLaunchKernelGGL((k_few<T, 1, 16, 1, ROWS_HELD, GRADIENT>), grid, threads, 0, stream, p); break;
    case kFourShort:
      if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((k_few<T, 4, 1, 4, ROWS_HELD, GRADIENT>), grid, threads, 0, stream, p);
      break;
    default:
      if constexpr (sizeof(T) == 4) hipLaunchKernelGGL((k_few<T, 4, 4, 2, ROWS_HELD, GRADIENT>), grid, threads, 0, stream, p);
      break;
  }
  return launched(what);
}

}  // namespace few

#endif  // SDNN_FEW_H
