// Layer norm of rows (gd_layer_norm_forward, gd_layer_norm_backward).
//
// Bound by the bytes.  Forward: a row is read once and waits in registers, as it lies in memory, until its statistics are known: up to
// 64 elements a thread, so that a warp has rows of up to 2048, or several short ones, by itself; weight and bias lie in shared memory; the next row's
// pieces are copied into shared memory by the threads that take them meanwhile.  The variance is the sum of squares about the mean, a second
// sum over the registers, not a difference of large numbers.  (32768 x 4096 in bf16: 98 us = 5.5 TB/s; 300000 x 64 22 us, 65 with a
// warp to each row; 8000 x 8192 58 us, 74 with 16 elements to a thread: instructions, 19 an element there, and not bytes were the time.)
//
// Backward: each thread keeps the sums of its columns, 16 of each gradient, which is why a row is spread over 4 .. 512 threads there.
#include <algorithm>
#include <cstring>

#include "gd_layers.cuh"
#include "gd_mma.cuh"

namespace gd {
namespace {

constexpr int kEach = 16;                      // backward: elements of a row a thread holds
constexpr uint32_t kMostThreads = 1024;
constexpr uint32_t kHeldWidth = 8192;                      // longer rows are read again for every sum
constexpr uint32_t kColumnCtas = 296;         // most CTAs that hold sums of columns

struct NormArgs {
  const void* x;
  const void* weight;
  const void* bias;
  void* y;
  float* mean;
  float* rstd;
  uint64_t ldx, ldy;
  uint32_t rows, width;
  float eps;
  uint32_t wide_params;                       // weight and bias are fp32
};
struct NormBackArgs {
  const void* dy;
  const void* x;
  const void* weight;
  const void* add;
  const float* mean;
  const float* rstd;
  void* dx;
  float* part;                                // [ctas][2][width], or NULL: no sums of columns are wanted
  float* dweight;                             // where they end: written here where the launch is one cluster
  float* dbias;
  uint32_t cluster, accumulate;
  uint64_t ld_dy, ldx, ld_add, ld_dx;
  uint32_t rows, width;
  uint32_t wide_params;
};

__device__ __forceinline__ uint64_t row_at(uint32_t r, uint64_t ld) { return r * ld; }
template <int DT>
__device__ __forceinline__ float param(const void* p, uint32_t i, uint32_t wide) {
  return wide ? static_cast<const float*>(p)[i] : Elem<DT>::get(static_cast<const typename Elem<DT>::type*>(p)[i]);
}

template <int G>
constexpr int kGroupThreads = G > 256 ? G : 256;       // of a CTA: one group, or several side by side

// Sum over a group's N values each; every thread of it gets the same.  `turn` alternates between calls: one barrier each suffices.
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&s)[N], float (*place)[N], uint32_t turn) {
#pragma unroll
  for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) s[i] += __shfl_xor_sync(0xFFFFFFFFu, s[i], o);
  }
  if constexpr (G > 32) {
    constexpr int W = G / 32;
    const uint32_t group = threadIdx.x / G;
    float(*at)[N] = place + (group * 2u + (turn & 1u)) * W;
    if ((threadIdx.x & 31u) == 0u) {
#pragma unroll
      for (int i = 0; i < N; ++i) at[(threadIdx.x % G) >> 5][i] = s[i];
    }
    if constexpr (G > 256) __syncthreads();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1u), "n"(G) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
      float t = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) t += at[w][i];
      s[i] = t;
    }
  }
}
template <int G>
constexpr int kSumPlaces = G > 32 ? 2 * kGroupThreads<G> / 32 : 1;

template <int G>
__device__ __forceinline__ void group_barrier() {
  if constexpr (G <= 32) __syncwarp();
  else if constexpr (G > 256) __syncthreads();
  else asm volatile("bar.sync %0, %1;" ::"r"(threadIdx.x / G + 1u), "n"(G) : "memory");
}

// The rows of `INPUTS` matrices, a few under way in shared memory.  A thread asks for and reads its own pieces, so nobody else waits.  Rows that
// start at odd multiples of two bytes (V = 1, 16 bits) are copied as the words that lie whole within them, each thread some, in places that keep
// their alignment; the elements that are left at the ends come through registers, a row ahead, and the group meets before it reads.
template <int DT, int V, int G, int INPUTS>
struct RowsAhead {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  static constexpr int kPieces = kEach / V, kBytes = V * (int)sizeof(T), kThreads = kGroupThreads<G>;
  static constexpr bool kWords = kBytes == 2;
  // as many as let two CTAs of 256 threads, or one of 512, have their place on an SM
  static constexpr uint32_t kDepth = sizeof(T) == 4 ? 2 : kThreads == 256 ? 3 : 4, kRowBytes = G * kEach * 2 + 16;
  static constexpr uint32_t kSmem = kDepth * INPUTS * (kWords ? kThreads / G * kRowBytes : kPieces * kThreads * kBytes);
  const T* from[INPUTS];
  uint64_t ld[INPUTS];
  uint32_t tid, rows, width;
  unsigned char* smem;
  T edge[INPUTS];
  __device__ __forceinline__ unsigned char* place(uint32_t slot, int input, int j) const {
    if constexpr (kWords) return smem + ((slot * INPUTS + input) * (kThreads / G) + threadIdx.x / G) * kRowBytes;
    else return smem + (((slot * INPUTS + input) * kPieces + j) * kThreads + threadIdx.x) * kBytes;
  }
  // 1 where a row starts between two words
  __device__ __forceinline__ uint32_t odd(int input, uint32_t row) const { return ((uint32_t)((uintptr_t)from[input] >> 1) ^ (row & (uint32_t)ld[input])) & 1u; }
  __device__ __forceinline__ void ask(uint32_t row, uint32_t slot) {
#pragma unroll
    for (int input = 0; input < INPUTS; ++input) {
      if (row >= rows || !from[input]) continue;
      const T* p = from[input] + row * ld[input];
      if constexpr (kWords) {
        const uint32_t o = odd(input, row), words = (width - o) / 2;
        const uint32_t to = smem_u32(place(slot, input, 0)) + 4u * o;
#pragma unroll
        for (int j = 0; j < kEach / 2; ++j) {
          const uint32_t k = tid + j * G;
          if (k < words) copy_ahead<4>(to + 4u * k, p + o + 2 * k);
        }
      } else {
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
          const uint32_t c = (tid + j * G) * V;
          if (c < width) copy_ahead<kBytes>(smem_u32(place(slot, input, j)), p + c);
        }
      }
    }
    copies_commit();
  }
  // the ends of the row that is taken next: the first element by thread 0, the last by thread 1
  __device__ __forceinline__ void ask_edges(uint32_t row) {
    if constexpr (kWords) {
#pragma unroll
      for (int input = 0; input < INPUTS; ++input) {
        if (row >= rows || !from[input]) continue;
        const T* p = from[input] + row * ld[input];
        const uint32_t o = odd(input, row);
        if (tid == 0 && o) edge[input] = p[0];
        if (tid == 1 && ((width - o) & 1u)) edge[input] = p[width - 1];
      }
    }
  }
  // the row in `slot` may be taken afterwards
  __device__ __forceinline__ void settle(uint32_t row, uint32_t slot) {
    copies_wait<(int)kDepth - 1>();
    if constexpr (kWords) {
#pragma unroll
      for (int input = 0; input < INPUTS; ++input) {
        if (row >= rows || !from[input]) continue;
        const uint32_t o = odd(input, row);
        T* to = reinterpret_cast<T*>(place(slot, input, 0)) + o;
        if (tid == 0 && o) to[0] = edge[input];
        if (tid == 1 && ((width - o) & 1u)) to[width - 1] = edge[input];
      }
      group_barrier<G>();
    }
  }
  // x: the row's elements (0 where there are none)
  __device__ __forceinline__ void take(uint32_t row, uint32_t slot, int input, float* x) const {
    const bool there = row < rows && from[input];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const uint32_t c = (tid + j * G) * V;
      typename P::Raw r = P::none();
      if (there && c < width) {
        if constexpr (kWords) r = reinterpret_cast<const typename P::Raw*>(place(slot, input, 0))[odd(input, row) + c];
        else r = *reinterpret_cast<const typename P::Raw*>(place(slot, input, j));
      }
      P::widen(r, x + j * V);
    }
  }
};

// ---------------------------------------------------------------- forward
// E elements of a row to each of G threads, held as they lie; G > 32: groups of a CTA meet at barriers of their own.
template <int DT, int V, int E, int G>
struct RowShape {
  using T = typename Elem<DT>::type;
  static constexpr int kPieces = E / V, kBytes = V * (int)sizeof(T), kThreads = 256;
  static constexpr bool kCopies = kBytes >= 4;         // (pieces of two bytes cannot be copied ahead)
  static constexpr uint32_t kSmem = kCopies ? kPieces * kBytes * kThreads : 0;      // weight and bias come behind this
};
// two neighbours (or one and a zero) of a piece
template <int DT, int V>
__device__ __forceinline__ float2 pair_of(const typename Piece<DT, V>::Raw& r, int i) {
  if constexpr (V == 1) {
    float x;
    Piece<DT, V>::widen(r, &x);
    return make_float2(x, 0.f);
  } else if constexpr (DT == GD_DTYPE_FP32) {
    const float* f = reinterpret_cast<const float*>(&r);
    return make_float2(f[2 * i], f[2 * i + 1]);
  } else {
    return unpack2<DT>(reinterpret_cast<const uint32_t*>(&r)[i]);
  }
}
template <int DT, int V, int E, int G>
__global__ void __launch_bounds__(RowShape<DT, V, E, G>::kThreads, E <= 32 ? 3 : 2) norm_kernel(const __grid_constant__ NormArgs a) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  using S = RowShape<DT, V, E, G>;
  constexpr int kPieces = S::kPieces, kGroups = S::kThreads / G, kPairs = V == 1 ? 1 : V / 2;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_sum[G > 32 ? 2 * S::kThreads / 32 : 1][1];
  float *s_w = reinterpret_cast<float*>(smem + S::kSmem), *s_b = s_w + (a.width + 3u & ~3u);
  const uint32_t tid = threadIdx.x % G;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  pdl_wait();
  pdl_trigger();
  // pieces of a row this thread has: the first `mine` of kPieces
  const uint32_t whole = a.width / V, mine = tid < whole ? (whole - tid + G - 1) / G : 0u;
  const uint32_t at = smem_u32(smem) + threadIdx.x * S::kBytes;
  const auto ask = [&](uint32_t row) {
    if constexpr (S::kCopies) {
      if (row < a.rows) {
        const T* from = x + row * a.ldx + tid * V;
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
          if (j < (int)mine) copy_ahead<S::kBytes>(at + j * (S::kThreads * S::kBytes), from + j * G * V);
      }
      copies_commit();
    }
  };
  const uint32_t step = gridDim.x * kGroups;
  uint32_t r = blockIdx.x * kGroups + threadIdx.x / G, turn = 0;
  ask(r);
  for (uint32_t c = threadIdx.x; c < a.width; c += S::kThreads) {
    s_w[c] = a.weight ? param<DT>(a.weight, c, a.wide_params) : 1.f;
    s_b[c] = a.bias ? param<DT>(a.bias, c, a.wide_params) : 0.f;
  }
  __syncthreads();
  const float count = (float)a.width;
  // (the groups of a warp stay together: those behind the last row go through the motions)
  for (uint32_t first = blockIdx.x * kGroups + (G < 32 ? threadIdx.x / 32 * (32 / G) : threadIdx.x / G); first < a.rows; first += step, r += step) {
    const bool live = r < a.rows;
    typename P::Raw raw[kPieces];
    if constexpr (S::kCopies) copies_wait<0>();
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      raw[j] = P::none();
      if (j < (int)mine && live) {
        if constexpr (S::kCopies) raw[j] = *reinterpret_cast<const typename P::Raw*>(smem + threadIdx.x * S::kBytes + j * (S::kThreads * S::kBytes));
        else raw[j] = P::load(x + row_at(r, a.ldx) + (tid + j * G) * V);
      }
    }
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
#pragma unroll
      for (int i = 0; i < kPairs; ++i) sum = add2(sum, pair_of<DT, V>(raw[j], i));
    }
    float s[1] = {sum.x + sum.y};
    group_sum<G>(s, s_sum, turn++);
    ask(r + step);                                     // (the sum has this row's values: they have been read)
    const float mean = s[0] / count;                   // (a product with 1 / count would not give a constant row's value back)
    const float2 less = both(-mean);
    sum = make_float2(0.f, 0.f);
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      if (j < (int)mine) {
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          float2 d = add2(pair_of<DT, V>(raw[j], i), less);
          if constexpr (V == 1) d.y = 0.f;
          sum = fma2(d, d, sum);
        }
      }
    }
    s[0] = sum.x + sum.y;
    group_sum<G>(s, s_sum, turn++);
    const float rstd = __frsqrt_rn(s[0] / count + a.eps);
    if (!live) continue;
    if (tid == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    T* to = y + row_at(r, a.ldy) + tid * V;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      if (j < (int)mine) {
        const uint32_t c = (tid + j * G) * V;
        float w[V], b[V], o[V];
        if constexpr (V >= 4) {
#pragma unroll
          for (int i = 0; i < V; i += 4) {
            const float4 p = *reinterpret_cast<const float4*>(s_w + c + i), q = *reinterpret_cast<const float4*>(s_b + c + i);
            w[i] = p.x, w[i + 1] = p.y, w[i + 2] = p.z, w[i + 3] = p.w, b[i] = q.x, b[i + 1] = q.y, b[i + 2] = q.z, b[i + 3] = q.w;
          }
        } else {
#pragma unroll
          for (int i = 0; i < V; ++i) w[i] = s_w[c + i], b[i] = s_b[c + i];
        }
#pragma unroll
        for (int i = 0; i < kPairs; ++i) {
          const float2 d = mul2(add2(pair_of<DT, V>(raw[j], i), less), both(rstd));
          if constexpr (V == 1) {
            o[0] = fmaf(d.x, w[0], b[0]);
          } else {
            const float2 e = fma2(d, make_float2(w[2 * i], w[2 * i + 1]), make_float2(b[2 * i], b[2 * i + 1]));
            o[2 * i] = e.x, o[2 * i + 1] = e.y;
          }
        }
        P::store(to + j * G * V, P::narrow(o));
      }
    }
  }
  if constexpr (S::kCopies) copies_wait<0>();
}

// Rows longer than the registers of a CTA: read once per sum and once for the result, from L2 after the first time.
template <int DT>
__global__ void __launch_bounds__(kMostThreads) norm_long_kernel(const __grid_constant__ NormArgs a) {
  using T = typename Elem<DT>::type;
  __shared__ float s_sum[2 * kMostThreads / 32][1];
  pdl_wait();
  pdl_trigger();
  uint32_t turn = 0;
  for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T* x = static_cast<const T*>(a.x) + r * a.ldx;
    T* y = static_cast<T*>(a.y) + r * a.ldy;
    float s[1] = {0.f};
#pragma unroll 4
    for (uint32_t c = threadIdx.x; c < a.width; c += kMostThreads) s[0] += Elem<DT>::get(x[c]);
    group_sum<(int)kMostThreads>(s, s_sum, turn++);
    const float mean = s[0] / (float)a.width;
    s[0] = 0.f;
#pragma unroll 4
    for (uint32_t c = threadIdx.x; c < a.width; c += kMostThreads) {
      const float e = Elem<DT>::get(x[c]) - mean;
      s[0] = fmaf(e, e, s[0]);
    }
    group_sum<(int)kMostThreads>(s, s_sum, turn++);
    const float rstd = __frsqrt_rn(s[0] / (float)a.width + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
    // (y may be x: each thread reads what it overwrites itself)
    for (uint32_t c = threadIdx.x; c < a.width; c += kMostThreads) {
      const float w = a.weight ? param<DT>(a.weight, c, a.wide_params) : 1.f, b = a.bias ? param<DT>(a.bias, c, a.wide_params) : 0.f;
      y[c] = Elem<DT>::put(fmaf((Elem<DT>::get(x[c]) - mean) * rstd, w, b));
    }
  }
}

// ---------------------------------------------------------------- backward
// A group's rows give dx; each thread keeps the sums of its columns, which meet in shared memory where a CTA has several groups and go to the
// workspace, a row of sums per CTA, to be joined in order by the next launch.
template <int DT, int V, int G>
__global__ void __launch_bounds__(kGroupThreads<G>, kGroupThreads<G> == 256 ? 2 : 1) norm_back_kernel(const __grid_constant__ NormBackArgs a) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  using Rows = RowsAhead<DT, V, G, 3>;
  constexpr int kPieces = kEach / V, kGroups = kGroupThreads<G> / G;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_sum[kSumPlaces<G>][2];
  __shared__ float s_part[kGroups][kGroups > 1 ? G * kEach : 1];
  const uint32_t tid = threadIdx.x % G;
  T* dx = static_cast<T*>(a.dx);
  pdl_wait();
  pdl_trigger();
  Rows in;
  in.from[0] = static_cast<const T*>(a.x), in.ld[0] = a.ldx;
  in.from[1] = static_cast<const T*>(a.dy), in.ld[1] = a.ld_dy;
  in.from[2] = static_cast<const T*>(a.add), in.ld[2] = a.ld_add;
  in.tid = tid, in.rows = a.rows, in.width = a.width, in.smem = smem;
  const uint32_t step = gridDim.x * kGroups;
  uint32_t r = blockIdx.x * kGroups + threadIdx.x / G, turn = 0, slot = 0;
#pragma unroll
  for (uint32_t n = 0; n < Rows::kDepth; ++n) in.ask(r + n * step, n);
  in.ask_edges(r);
  float next_mean = r < a.rows ? a.mean[r] : 0.f, next_rstd = r < a.rows ? a.rstd[r] : 0.f;
  float w[kEach], dw[kEach], db[kEach];
#pragma unroll
  for (int j = 0; j < kPieces; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t c = (tid + j * G) * V + i;
      w[j * V + i] = a.weight && c < a.width ? param<DT>(a.weight, c, a.wide_params) : 1.f;
      dw[j * V + i] = db[j * V + i] = 0.f;
    }
  }
  const float share = 1.f / (float)a.width;
  // (the groups of a warp stay together: those behind the last row go through the motions)
  for (uint32_t first = blockIdx.x * kGroups + (G < 32 ? threadIdx.x / 32 * (32 / G) : threadIdx.x / G); first < a.rows; first += step, r += step) {
    float n[kEach], g[kEach], more[kEach];
    const float mean = next_mean, rstd = next_rstd;
    in.settle(r, slot);
    in.take(r, slot, 0, n);
    in.take(r, slot, 1, g);
    if constexpr (Rows::kWords) in.take(r, slot, 2, more);         // (others copy into its place: read before the group meets)
    in.ask_edges(r + step);
    if (r + step < a.rows) next_mean = a.mean[r + step], next_rstd = a.rstd[r + step];
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const bool there = (tid + j * G) * V < a.width;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = j * V + i;
        n[e] = there ? (n[e] - mean) * rstd : 0.f;
        dw[e] = fmaf(g[e], n[e], dw[e]);
        db[e] += g[e];
        g[e] *= w[e];
        s[0] += g[e];
        s[1] = fmaf(g[e], n[e], s[1]);
      }
    }
    if (a.dx) {
      group_sum<G>(s, s_sum, turn++);
      const float m0 = s[0] * share, m1 = s[1] * share;
      if constexpr (!Rows::kWords) in.take(r, slot, 2, more);
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        const uint32_t c = (tid + j * G) * V;
        if (c < a.width && r < a.rows) {
          float o[V];
#pragma unroll
          for (int i = 0; i < V; ++i) o[i] = fmaf(g[j * V + i] - m0 - n[j * V + i] * m1, rstd, more[j * V + i]);
          P::store(dx + r * a.ld_dx + c, P::narrow(o));
        }
      }
    }
    if (Rows::kWords && (G <= 32 || !a.dx)) group_barrier<G>();    // (all have read; else the sum's barrier says so)
    in.ask(r + Rows::kDepth * step, slot);
    if (++slot == Rows::kDepth) slot = 0;
  }
  copies_wait<0>();
  if (!a.part) return;
  // the CTA's sums of columns, in the rows' place
  float* sums = reinterpret_cast<float*>(smem);
  static_assert(Rows::kSmem >= 2 * G * kEach * 4, "two sums for every column");
  if constexpr (kGroups > 1) {
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      const float* t = pass ? db : dw;
      __syncthreads();
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
#pragma unroll
        for (int i = 0; i < V; ++i) s_part[threadIdx.x / G][(tid + j * G) * V + i] = t[j * V + i];
      }
      __syncthreads();
      for (uint32_t c = threadIdx.x; c < a.width; c += kGroupThreads<G>) {
        float q = 0.f;
#pragma unroll 8
        for (int group = 0; group < kGroups; ++group) q += s_part[group][c];
        sums[pass * a.width + c] = q;
      }
    }
  } else {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const uint32_t c = (tid + j * G) * V + i;
        if (c < a.width) sums[c] = dw[j * V + i], sums[a.width + c] = db[j * V + i];
      }
    }
  }
  // the cluster's, in rank order, each CTA a share of the columns
  const bool clustered = a.cluster > 1, last = gridDim.x == a.cluster;
  const uint32_t rank = clustered ? cluster_rank() : 0u;
  if (clustered) {
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
  float* part = a.part + (uint64_t)blockIdx.x * 2 * a.width;         // (a cluster is the whole launch)
  for (uint32_t c = rank * kGroupThreads<G> + threadIdx.x; c < 2 * a.width; c += a.cluster * kGroupThreads<G>) {
    float q = 0.f;
    if (clustered) {
      const uint32_t at = smem_u32(sums + c);
      for (uint32_t n = 0; n < a.cluster; ++n) q += peer_load1(peer_address(at, n));
    } else {
      q = sums[c];
    }
    if (!last) {
      part[c] = q;
    } else {
      float* to = c < a.width ? a.dweight : a.dbias;
      const uint32_t at = c < a.width ? c : c - a.width;
      if (to) to[at] = a.accumulate ? to[at] + q : q;
    }
  }
  if (clustered) {
    cluster_arrive();                                  // (the others may still be reading this CTA's sums)
    cluster_wait();
  }
}

// Long rows: sums and dx from memory, the sums of columns by a launch of their own.
template <int DT>
__global__ void __launch_bounds__(kMostThreads) norm_back_long_kernel(const __grid_constant__ NormBackArgs a) {
  using T = typename Elem<DT>::type;
  __shared__ float s_sum[2 * kMostThreads / 32][2];
  pdl_wait();
  pdl_trigger();
  uint32_t turn = 0;
  for (uint32_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const T *x = static_cast<const T*>(a.x) + r * a.ldx, *dy = static_cast<const T*>(a.dy) + r * a.ld_dy;
    const T* add = a.add ? static_cast<const T*>(a.add) + r * a.ld_add : nullptr;
    T* dx = static_cast<T*>(a.dx) + r * a.ld_dx;
    const float mean = a.mean[r], rstd = a.rstd[r];
    float s[2] = {0.f, 0.f};
#pragma unroll 2
    for (uint32_t c = threadIdx.x; c < a.width; c += kMostThreads) {
      const float g = Elem<DT>::get(dy[c]) * (a.weight ? param<DT>(a.weight, c, a.wide_params) : 1.f);
      s[0] += g;
      s[1] = fmaf(g, (Elem<DT>::get(x[c]) - mean) * rstd, s[1]);
    }
    group_sum<(int)kMostThreads>(s, s_sum, turn++);
    const float m0 = s[0] / (float)a.width, m1 = s[1] / (float)a.width;
    for (uint32_t c = threadIdx.x; c < a.width; c += kMostThreads) {
      const float g = Elem<DT>::get(dy[c]) * (a.weight ? param<DT>(a.weight, c, a.wide_params) : 1.f);
      float o = (g - m0 - (Elem<DT>::get(x[c]) - mean) * rstd * m1) * rstd;
      if (add) o += Elem<DT>::get(add[c]);
      dx[c] = Elem<DT>::put(o);
    }
  }
}
constexpr uint32_t kLongColumnThreads = 256;
template <int DT>
__global__ void __launch_bounds__(kLongColumnThreads) norm_long_columns_kernel(const __grid_constant__ NormBackArgs a) {
  using T = typename Elem<DT>::type;
  pdl_wait();
  pdl_trigger();
  const uint32_t c = blockIdx.x * kLongColumnThreads + threadIdx.x;
  if (c >= a.width) return;
  const T *x = static_cast<const T*>(a.x) + c, *dy = static_cast<const T*>(a.dy) + c;
  float dw = 0.f, db = 0.f;
#pragma unroll 4
  for (uint32_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const float g = Elem<DT>::get(dy[r * a.ld_dy]);
    dw = fmaf(g, (Elem<DT>::get(x[r * a.ldx]) - a.mean[r]) * a.rstd[r], dw);
    db += g;
  }
  float* part = a.part + (uint64_t)blockIdx.y * 2 * a.width + c;
  part[0] = dw, part[a.width] = db;
}

// The CTAs' sums, joined in order: a warp's lanes are 32 columns, the warps share the CTAs.
constexpr uint32_t kJoinWarps = 32, kJoinInHand = (kColumnCtas + kJoinWarps - 1) / kJoinWarps;      // all of a warp's loads at once
__global__ void __launch_bounds__(32 * kJoinWarps) norm_join_kernel(const float* part, uint32_t ctas, uint32_t width, float* dweight, float* dbias, uint32_t accumulate) {
  __shared__ float s_sum[kJoinWarps][33];
  pdl_wait();
  pdl_trigger();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, c = blockIdx.x * 32u + lane, which = blockIdx.y;
  float* out = which ? dbias : dweight;
  if (!out) return;
  float s = 0.f;
  if (c < width) {
    float x[kJoinInHand];
#pragma unroll
    for (uint32_t u = 0; u < kJoinInHand; ++u) {
      const uint32_t q = warp + u * kJoinWarps;
      x[u] = q < ctas ? part[((uint64_t)q * 2 + which) * width + c] : 0.f;
    }
#pragma unroll
    for (uint32_t u = 0; u < kJoinInHand; ++u) s += x[u];
  }
  s_sum[warp][lane] = s;
  __syncthreads();
  if (warp == 0 && c < width) {
    float t = 0.f;
#pragma unroll
    for (uint32_t q = 0; q < kJoinWarps; ++q) t += s_sum[q][lane];
    out[c] = accumulate ? out[c] + t : t;
  }
}

// ---------------------------------------------------------------- host side
// How many CTAs of a kernel an SM holds, asked once.
template <typename Kernel>
cudaError_t resident_ctas(Kernel kernel, PerDeviceInt& held, uint32_t threads, uint32_t smem, uint32_t* per_sm) {
  int dev, n = held.get(&dev);
  if (!n) {
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, (int)threads, smem);
    if (e != cudaSuccess) return e;
    n = std::max(n, 1);
    held.set(dev, n);
  }
  *per_sm = (uint32_t)n;
  return cudaSuccess;
}
template <int DT, int V, int E, int G>
cudaError_t launch_forward(const NormArgs& a, cudaStream_t stream) {
  using S = RowShape<DT, V, E, G>;
  constexpr uint32_t kMost = S::kSmem + 2 * E * G * 4, kGroups = S::kThreads / G;      // with the parameters of the widest row
  const uint32_t smem = S::kSmem + 2 * (a.width + 3u & ~3u) * 4;
  auto kernel = norm_kernel<DT, V, E, G>;
  static PerDeviceInt held;
  uint32_t per_sm;
  const cudaError_t e = resident_ctas(kernel, held, S::kThreads, kMost, &per_sm);
  if (e != cudaSuccess) return e;
  return launch_dependent(kernel, dim3(std::min((a.rows + kGroups - 1) / kGroups, (uint32_t)sm_count() * per_sm)), dim3(S::kThreads), smem, stream, a);
}
// A launch that fits one cluster ends the sums itself (*ctas = 0: nothing is left to join); others leave a row of sums per CTA.  (In clusters of four,
// which left a quarter of the rows to join, 16384 x 4096 took 125 us in place of 87.)
constexpr uint32_t kOneCluster = 8, kOneRows = 3;      // kOneRows: rows a group takes rather than have a launch join the sums
template <int DT, int V, int G>
cudaError_t launch_backward(NormBackArgs a, uint32_t* ctas, cudaStream_t stream) {
  constexpr uint32_t threads = kGroupThreads<G>, groups = threads / G, smem = RowsAhead<DT, V, G, 3>::kSmem;
  auto kernel = norm_back_kernel<DT, V, G>;
  static PerDeviceInt held;
  uint32_t per_sm;
  cudaError_t e = resident_ctas(kernel, held, threads, smem, &per_sm);
  if (e != cudaSuccess) return e;
  const uint32_t want = (a.rows + groups - 1) / groups;
  uint32_t grid = std::min(want, std::min(kColumnCtas, (uint32_t)sm_count() * per_sm));
  a.cluster = 1;
  if (a.part && want <= kOneCluster * kOneRows) {
    while (a.cluster < kOneCluster && a.cluster < want) a.cluster *= 2;
    grid = a.cluster;
  }
  *ctas = grid == a.cluster ? 0 : grid;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.cluster > 1 ? 2 : 1;
  ProfileScope ps(stream, PT_NORM_BACK);
  e = cudaLaunchKernelEx(&cfg, kernel, a);
  if (e == cudaSuccess) note_launches(1);
  return e;
}
// Up to 64 elements to a thread, so that what a row costs beside its elements is shared by many, and eight threads at least, so that they read whole
// lines.  Single elements of 16 bits take a register each: half as many (20000 x 1001: 26 against 35 us).
template <int DT, int V>
cudaError_t forward_v(const NormArgs& a, cudaStream_t stream) {
  const uint32_t width = a.width;
  if (width <= 8 * 8) return launch_forward<DT, V, 8, 8>(a, stream);
  if (width <= 8 * 32) return launch_forward<DT, V, 32, 8>(a, stream);
  if constexpr (V == 1) {
    if (width <= 32 * 32) return launch_forward<DT, V, 32, 32>(a, stream);
    if (width <= 64 * 32) return launch_forward<DT, V, 32, 64>(a, stream);
    return launch_forward<DT, V, 32, 256>(a, stream);
  } else {
    if (width <= 8 * 64) return launch_forward<DT, V, 64, 8>(a, stream);
    if (width <= 16 * 64) return launch_forward<DT, V, 64, 16>(a, stream);
    if (width <= 32 * 64) return launch_forward<DT, V, 64, 32>(a, stream);
    if (width <= 64 * 64) return launch_forward<DT, V, 64, 64>(a, stream);
    return launch_forward<DT, V, 64, 128>(a, stream);
  }
}
// backward: threads per row, kEach elements each
template <int DT, int V>
cudaError_t backward_v(const NormBackArgs& a, uint32_t* ctas, cudaStream_t stream) {
  const uint32_t width = a.width;
  if (width <= 4 * kEach) return launch_backward<DT, V, 4>(a, ctas, stream);
  if (width <= 16 * kEach) return launch_backward<DT, V, 16>(a, ctas, stream);
  if (width <= 32 * kEach) return launch_backward<DT, V, 32>(a, ctas, stream);
  if (width <= 64 * kEach) return launch_backward<DT, V, 64>(a, ctas, stream);
  if (width <= 128 * kEach) return launch_backward<DT, V, 128>(a, ctas, stream);
  if (width <= 256 * kEach) return launch_backward<DT, V, 256>(a, ctas, stream);
  return launch_backward<DT, V, 512>(a, ctas, stream);
}

template <int DT>
cudaError_t forward_t(const NormArgs& a, cudaStream_t stream) {
  constexpr size_t item = sizeof(typename Elem<DT>::type);
  if (a.width > kHeldWidth)
    return launch_dependent(norm_long_kernel<DT>, dim3(std::min(a.rows, 2u * (uint32_t)sm_count())), dim3(kMostThreads), 0, stream, a);
  const auto takes = [&](uint32_t v) { return in_pieces(a.x, a.ldx, a.rows, a.width, item, v) && in_pieces(a.y, a.ldy, a.rows, a.width, item, v); };
  if constexpr (item == 4) {
    return takes(4) ? forward_v<DT, 4>(a, stream) : forward_v<DT, 1>(a, stream);
  } else {
    return takes(8) ? forward_v<DT, 8>(a, stream) : takes(4) ? forward_v<DT, 4>(a, stream) : forward_v<DT, 1>(a, stream);
  }
}
template <int DT>
cudaError_t backward_t(const NormBackArgs& a, uint32_t* ctas, cudaStream_t stream) {
  constexpr size_t item = sizeof(typename Elem<DT>::type);
  if (a.width > kHeldWidth) {
    if (a.part) {      // (first: dx may take dy's place)
      const uint32_t across = (a.width + kLongColumnThreads - 1) / kLongColumnThreads;
      *ctas = std::min(a.rows, std::min(kColumnCtas, std::max(1u, 4u * (uint32_t)sm_count() / across)));
      ProfileScope ps(stream, PT_NORM_BACK);
      const cudaError_t e = launch_dependent(norm_long_columns_kernel<DT>, dim3(across, *ctas), dim3(kLongColumnThreads), 0, stream, a);
      if (e != cudaSuccess) return e;
      note_launches(1);
    }
    if (!a.dx) return cudaSuccess;
    ProfileScope ps(stream, PT_NORM_BACK);
    const cudaError_t e = launch_dependent(norm_back_long_kernel<DT>, dim3(std::min(a.rows, 2u * (uint32_t)sm_count())), dim3(kMostThreads), 0, stream, a);
    if (e == cudaSuccess) note_launches(1);
    return e;
  }
  const auto takes = [&](uint32_t v) {
    return in_pieces(a.x, a.ldx, a.rows, a.width, item, v) && in_pieces(a.dy, a.ld_dy, a.rows, a.width, item, v) &&
           in_pieces(a.add, a.ld_add, a.rows, a.width, item, v) && in_pieces(a.dx, a.ld_dx, a.rows, a.width, item, v);
  };
  if constexpr (item == 4) {
    return takes(4) ? backward_v<DT, 4>(a, ctas, stream) : backward_v<DT, 1>(a, ctas, stream);
  } else {
    return takes(8) ? backward_v<DT, 8>(a, ctas, stream) : takes(4) ? backward_v<DT, 4>(a, ctas, stream) : backward_v<DT, 1>(a, ctas, stream);
  }
}

int check_shape(uint64_t rows, uint64_t width, int dtype, int param_dtype, bool params) {
  if (!is_dtype(dtype) || (params && param_dtype != dtype && param_dtype != GD_DTYPE_FP32) || width == 0) return GD_ERR_INVALID_ARG;
  return rows >> 31 || width >> 31 ? GD_ERR_TOO_LARGE : GD_OK;
}

int forward(const gd_layer_norm_forward_args* g, cudaStream_t stream) {
  if (!g || g->reserved != 0 || !(g->eps >= 0.f)) return GD_ERR_INVALID_ARG;
  const int rc = check_shape(g->rows, g->width, g->dtype, g->param_dtype, g->weight || g->bias);
  if (rc != GD_OK) return rc;
  if (g->rows == 0) return GD_OK;
  const size_t item = dtype_bytes(g->dtype), p_item = dtype_bytes(g->param_dtype);
  if (!good_matrix(g->x, g->ldx, g->rows, g->width, item) || !good_matrix(g->y, g->ldy, g->rows, g->width, item)) return GD_ERR_INVALID_ARG;
  if ((g->weight && !aligned_to(g->weight, p_item)) || (g->bias && !aligned_to(g->bias, p_item)) || !aligned_to(g->mean, 4) || !aligned_to(g->rstd, 4))
    return GD_ERR_INVALID_ARG;
  if (g->x == g->y && g->rows > 1 && g->ldx != g->ldy) return GD_ERR_INVALID_ARG;
  NormArgs a;
  std::memset(&a, 0, sizeof(a));
  a.x = g->x, a.ldx = g->ldx;
  a.y = g->y, a.ldy = g->ldy;
  a.weight = g->weight, a.bias = g->bias;
  a.mean = g->mean, a.rstd = g->rstd;
  a.rows = (uint32_t)g->rows, a.width = (uint32_t)g->width;
  a.eps = g->eps;
  a.wide_params = g->param_dtype == GD_DTYPE_FP32;
  ProfileScope ps(stream, PT_NORM);
  const cudaError_t e = g->dtype == GD_DTYPE_FP32   ? forward_t<GD_DTYPE_FP32>(a, stream)
                        : g->dtype == GD_DTYPE_BF16 ? forward_t<GD_DTYPE_BF16>(a, stream)
                                                    : forward_t<GD_DTYPE_FP16>(a, stream);
  if (e != cudaSuccess) return GD_ERR_CUDA;
  note_launches(1);
  return GD_OK;
}

int backward(const gd_layer_norm_backward_args* g, cudaStream_t stream) {
  if (!g || g->reserved != 0 || (g->flags & ~(uint32_t)GD_LAYER_NORM_ACCUMULATE)) return GD_ERR_INVALID_ARG;
  const int rc = check_shape(g->rows, g->width, g->dtype, g->param_dtype, g->weight != nullptr);
  if (rc != GD_OK) return rc;
  const bool has_dx = g->dx && g->rows, sums = g->dweight || g->dbias, accumulate = (g->flags & GD_LAYER_NORM_ACCUMULATE) != 0;
  if (!has_dx && !sums) return GD_OK;
  if (!aligned_to(g->dweight, 4) || !aligned_to(g->dbias, 4)) return GD_ERR_INVALID_ARG;
  const uint64_t rows = g->rows, width = g->width;
  const size_t item = dtype_bytes(g->dtype);
  if (rows) {
    if (!good_matrix(g->dy, g->ld_dy, rows, width, item) || !good_matrix(g->x, g->ldx, rows, width, item) || !g->mean || !g->rstd || !aligned_to(g->mean, 4) ||
        !aligned_to(g->rstd, 4) || (g->weight && !aligned_to(g->weight, dtype_bytes(g->param_dtype))))
      return GD_ERR_INVALID_ARG;
    if ((g->dx && !good_matrix(g->dx, g->ld_dx, rows, width, item)) || (g->add && !good_matrix(g->add, g->ld_add, rows, width, item))) return GD_ERR_INVALID_ARG;
    if (rows > 1 && g->dx && ((g->dx == g->dy && g->ld_dx != g->ld_dy) || (g->dx == g->add && g->ld_dx != g->ld_add))) return GD_ERR_INVALID_ARG;
  }
  NormBackArgs a;
  std::memset(&a, 0, sizeof(a));
  uint32_t ctas = 0;
  if (sums) {
    size_t need = 0;
    gd_layer_norm_workspace_bytes(rows, width, &need);
    if (!g->workspace || !aligned_to(g->workspace, 256) || g->workspace_bytes < need) return GD_ERR_WORKSPACE;
    a.part = static_cast<float*>(g->workspace);
    a.dweight = g->dweight, a.dbias = g->dbias;
    a.accumulate = accumulate;
  }
  if (rows) {
    a.dy = g->dy, a.ld_dy = g->ld_dy;
    a.x = g->x, a.ldx = g->ldx;
    a.add = g->dx ? g->add : nullptr, a.ld_add = g->ld_add;
    a.dx = g->dx, a.ld_dx = g->ld_dx;
    a.weight = g->weight;
    a.mean = g->mean, a.rstd = g->rstd;
    a.rows = (uint32_t)rows, a.width = (uint32_t)width;
    a.wide_params = g->param_dtype == GD_DTYPE_FP32;
    const cudaError_t e = g->dtype == GD_DTYPE_FP32   ? backward_t<GD_DTYPE_FP32>(a, &ctas, stream)
                          : g->dtype == GD_DTYPE_BF16 ? backward_t<GD_DTYPE_BF16>(a, &ctas, stream)
                                                      : backward_t<GD_DTYPE_FP16>(a, &ctas, stream);
    if (e != cudaSuccess) return GD_ERR_CUDA;
  }
  if (sums && (ctas || !rows)) {
    ProfileScope ps(stream, PT_NORM_JOIN);
    const cudaError_t e = launch_dependent(norm_join_kernel, dim3((uint32_t)((width + 31) / 32), 2), dim3(32 * kJoinWarps), 0, stream, (const float*)a.part, ctas,
                                           (uint32_t)width, g->dweight, g->dbias, (uint32_t)accumulate);
    if (e != cudaSuccess) return GD_ERR_CUDA;
    note_launches(1);
  }
  return GD_OK;
}

}  // namespace
}  // namespace gd

extern "C" {

int gd_layer_norm_workspace_bytes(uint64_t rows, uint64_t width, size_t* bytes_out) {
  if (!bytes_out) return GD_ERR_INVALID_ARG;
  if (rows >> 31 || width >> 31) return GD_ERR_TOO_LARGE;
  *bytes_out = (size_t)(std::max<uint64_t>(1, std::min<uint64_t>(rows, gd::kColumnCtas)) * 2 * width * 4);
  return GD_OK;
}
int gd_layer_norm_forward(const gd_layer_norm_forward_args* a, void* stream) { return gd::forward(a, (cudaStream_t)stream); }
int gd_layer_norm_backward(const gd_layer_norm_backward_args* a, void* stream) { return gd::backward(a, (cudaStream_t)stream); }

}  // extern "C"
