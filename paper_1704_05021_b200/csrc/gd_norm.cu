// Layer norm of rows (gd_layer_norm_forward, gd_layer_norm_backward).
//
// Bound by the bytes: a row is read once and waits in registers, kEach elements a thread, until its statistics are known.  A group of
// G threads holds a row: a warp (four rows a CTA then) or a whole CTA of 64 .. 512 threads; groups take rows in turn and ask for the next
// one before they work on this one.  The variance is the sum of squares about the mean, a second sum over the registers, not a
// difference of large numbers.
#include <algorithm>
#include <cstring>

#include "gd_layers.cuh"

namespace gd {
namespace {

constexpr int kEach = 16;                     // elements of a row a thread holds
constexpr uint32_t kMostThreads = 1024;
constexpr uint32_t kHeldWidth = kEach * 512;               // longer rows are read again for every sum
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
  uint64_t ld_dy, ldx, ld_add, ld_dx;
  uint32_t rows, width;
  uint32_t wide_params;
};

template <int DT>
__device__ __forceinline__ float param(const void* p, uint32_t i, uint32_t wide) {
  return wide ? static_cast<const float*>(p)[i] : Elem<DT>::get(static_cast<const typename Elem<DT>::type*>(p)[i]);
}

// Sum over a group's N values each; every thread of it gets the same.  `turn` alternates between calls: one barrier each suffices.
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&s)[N], float (*place)[N], uint32_t turn) {
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = warp_sum(s[i]);
  if constexpr (G > 32) {
    constexpr int W = G / 32;
    float(*at)[N] = place + (turn & 1u) * W;
    if ((threadIdx.x & 31u) == 0u) {
#pragma unroll
      for (int i = 0; i < N; ++i) at[threadIdx.x >> 5][i] = s[i];
    }
    __syncthreads();
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
constexpr int kGroupThreads = G > 32 ? G : 128;

// ---------------------------------------------------------------- forward
template <int DT, int V, int G>
__global__ void __launch_bounds__(kGroupThreads<G>) norm_kernel(const __grid_constant__ NormArgs a) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  constexpr int kPieces = kEach / V, kThreads = kGroupThreads<G>, kGroups = kThreads / G;
  __shared__ float s_sum[G > 32 ? 2 * G / 32 : 1][1];
  const uint32_t tid = threadIdx.x % G;
  const T* x = static_cast<const T*>(a.x);
  T* y = static_cast<T*>(a.y);
  pdl_wait();
  pdl_trigger();
  float w[kEach], b[kEach];
#pragma unroll
  for (int j = 0; j < kPieces; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t c = (tid + j * G) * V + i;
      w[j * V + i] = a.weight && c < a.width ? param<DT>(a.weight, c, a.wide_params) : 1.f;
      b[j * V + i] = a.bias && c < a.width ? param<DT>(a.bias, c, a.wide_params) : 0.f;
    }
  }
  const uint32_t step = gridDim.x * kGroups;
  uint32_t r = blockIdx.x * kGroups + threadIdx.x / G, turn = 0;
  typename P::Raw next[kPieces];
  const auto ask = [&](uint32_t row) {
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const uint32_t c = (tid + j * G) * V;
      next[j] = row < a.rows && c < a.width ? P::load(x + row * a.ldx + c) : P::none();
    }
  };
  ask(r);
  const float count = (float)a.width;
  for (; r < a.rows; r += step) {
    float v[kEach];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) P::widen(next[j], v + j * V);
    ask(r + step);
    float s[1] = {0.f};
#pragma unroll
    for (int j = 0; j < kEach; ++j) s[0] += v[j];
    group_sum<G>(s, s_sum, turn++);
    const float mean = s[0] / count;
    s[0] = 0.f;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const bool in = (tid + j * G) * V < a.width;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float& e = v[j * V + i];
        e -= mean;
        s[0] = in ? fmaf(e, e, s[0]) : s[0];
      }
    }
    group_sum<G>(s, s_sum, turn++);
    const float rstd = __frsqrt_rn(s[0] / count + a.eps);
    if (tid == 0) {
      if (a.mean) a.mean[r] = mean;
      if (a.rstd) a.rstd[r] = rstd;
    }
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const uint32_t c = (tid + j * G) * V;
      if (c < a.width) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[j * V + i] = fmaf(v[j * V + i] * rstd, w[j * V + i], b[j * V + i]);
        P::store(y + r * a.ldy + c, P::narrow(v + j * V));
      }
    }
  }
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
    group_sum<kMostThreads>(s, s_sum, turn++);
    const float mean = s[0] / (float)a.width;
    s[0] = 0.f;
#pragma unroll 4
    for (uint32_t c = threadIdx.x; c < a.width; c += kMostThreads) {
      const float e = Elem<DT>::get(x[c]) - mean;
      s[0] = fmaf(e, e, s[0]);
    }
    group_sum<kMostThreads>(s, s_sum, turn++);
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
// A group's rows give dx; each thread keeps the sums of its columns, which meet in shared memory (groups of a warp) and go to the
// workspace, a row of sums per CTA, to be joined in order by the next launch.
template <int DT, int V, int G>
__global__ void __launch_bounds__(kGroupThreads<G>) norm_back_kernel(const __grid_constant__ NormBackArgs a) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  constexpr int kPieces = kEach / V, kThreads = kGroupThreads<G>, kGroups = kThreads / G;
  __shared__ float s_sum[G > 32 ? 2 * G / 32 : 1][2];
  __shared__ float s_part[kGroups > 1 ? kGroups - 1 : 1][kGroups > 1 ? G * kEach : 1];
  const uint32_t tid = threadIdx.x % G;
  const T *x = static_cast<const T*>(a.x), *dy = static_cast<const T*>(a.dy), *add = static_cast<const T*>(a.add);
  T* dx = static_cast<T*>(a.dx);
  pdl_wait();
  pdl_trigger();
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
  const uint32_t step = gridDim.x * kGroups;
  uint32_t r = blockIdx.x * kGroups + threadIdx.x / G, turn = 0;
  typename P::Raw next_x[kPieces], next_g[kPieces];
  float next_mean = 0.f, next_rstd = 0.f;
  const auto ask = [&](uint32_t row) {
    const bool in = row < a.rows;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const uint32_t c = (tid + j * G) * V;
      next_x[j] = in && c < a.width ? P::load(x + row * a.ldx + c) : P::none();
      next_g[j] = in && c < a.width ? P::load(dy + row * a.ld_dy + c) : P::none();
    }
    next_mean = in ? a.mean[row] : 0.f;
    next_rstd = in ? a.rstd[row] : 0.f;
  };
  ask(r);
  const float share = 1.f / (float)a.width;
  for (; r < a.rows; r += step) {
    float n[kEach], g[kEach];
    typename P::Raw more[kPieces];
    const float mean = next_mean, rstd = next_rstd;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const uint32_t c = (tid + j * G) * V;
      P::widen(next_x[j], n + j * V);
      P::widen(next_g[j], g + j * V);
      if (add && a.dx && c < a.width) more[j] = P::load(add + r * a.ld_add + c);
    }
    ask(r + step);
    float s[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const bool in = (tid + j * G) * V < a.width;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int e = j * V + i;
        n[e] = in ? (n[e] - mean) * rstd : 0.f;
        dw[e] = fmaf(g[e], n[e], dw[e]);
        db[e] += g[e];
        g[e] *= w[e];
        s[0] += g[e];
        s[1] = fmaf(g[e], n[e], s[1]);
      }
    }
    if (!a.dx) continue;
    group_sum<G>(s, s_sum, turn++);
    const float m0 = s[0] * share, m1 = s[1] * share;
#pragma unroll
    for (int j = 0; j < kPieces; ++j) {
      const uint32_t c = (tid + j * G) * V;
      if (c < a.width) {
        float o[V], q[V];
        if (add) P::widen(more[j], q);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          o[i] = (g[j * V + i] - m0 - n[j * V + i] * m1) * rstd;
          if (add) o[i] += q[i];
        }
        P::store(dx + r * a.ld_dx + c, P::narrow(o));
      }
    }
  }
  if (!a.part) return;
  if constexpr (kGroups > 1) {
    const uint32_t group = threadIdx.x / G;
#pragma unroll
    for (int pass = 0; pass < 2; ++pass) {
      float* t = pass ? db : dw;
      __syncthreads();
      if (group) {
#pragma unroll
        for (int e = 0; e < kEach; ++e) s_part[group - 1][e * G + tid] = t[e];
      }
      __syncthreads();
      if (!group) {
        for (int q = 0; q < kGroups - 1; ++q) {
#pragma unroll
          for (int e = 0; e < kEach; ++e) t[e] += s_part[q][e * G + tid];
        }
      }
    }
    if (group) return;
  }
  float* part = a.part + (uint64_t)blockIdx.x * 2 * a.width;
#pragma unroll
  for (int j = 0; j < kPieces; ++j) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const uint32_t c = (tid + j * G) * V + i;
      if (c < a.width) part[c] = dw[j * V + i], part[a.width + c] = db[j * V + i];
    }
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
    group_sum<kMostThreads>(s, s_sum, turn++);
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
constexpr uint32_t kJoinWarps = 16;
__global__ void __launch_bounds__(32 * kJoinWarps) norm_join_kernel(const float* part, uint32_t ctas, uint32_t width, float* dweight, float* dbias, uint32_t accumulate) {
  __shared__ float s_sum[kJoinWarps][33];
  pdl_wait();
  pdl_trigger();
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, c = blockIdx.x * 32u + lane, which = blockIdx.y;
  float* out = which ? dbias : dweight;
  if (!out) return;
  float s = 0.f;
  if (c < width) {
#pragma unroll 8
    for (uint32_t q = warp; q < ctas; q += kJoinWarps) s += part[((uint64_t)q * 2 + which) * width + c];
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
// CTAs that fill the GPU, for a kernel of `threads` threads that takes `groups` rows at a time.
uint32_t row_ctas(uint32_t rows, uint32_t groups, uint32_t threads, uint32_t most) {
  const uint32_t want = (rows + groups - 1) / groups;
  return std::min(want, std::min(most, (uint32_t)sm_count() * std::max(1u, 1024u / threads)));
}
template <int DT, int V, int G>
cudaError_t launch_forward(const NormArgs& a, cudaStream_t stream) {
  constexpr uint32_t threads = kGroupThreads<G>;
  return launch_dependent(norm_kernel<DT, V, G>, dim3(row_ctas(a.rows, threads / G, threads, 0x7FFFFFFFu)), dim3(threads), 0, stream, a);
}
template <int DT, int V, int G>
cudaError_t launch_backward(const NormBackArgs& a, uint32_t* ctas, cudaStream_t stream) {
  constexpr uint32_t threads = kGroupThreads<G>;
  *ctas = row_ctas(a.rows, threads / G, threads, kColumnCtas);
  return launch_dependent(norm_back_kernel<DT, V, G>, dim3(*ctas), dim3(threads), 0, stream, a);
}
// threads per row: kEach elements each
#define GD_BY_WIDTH(CALL, ...)                                                         \
  (width <= 32 * kEach     ? CALL<DT, V, 32>(__VA_ARGS__)                              \
   : width <= 64 * kEach   ? CALL<DT, V, 64>(__VA_ARGS__)                              \
   : width <= 128 * kEach  ? CALL<DT, V, 128>(__VA_ARGS__)                             \
   : width <= 256 * kEach  ? CALL<DT, V, 256>(__VA_ARGS__)                             \
                           : CALL<DT, V, 512>(__VA_ARGS__))
template <int DT, int V>
cudaError_t forward_v(const NormArgs& a, cudaStream_t stream) {
  const uint32_t width = a.width;
  return GD_BY_WIDTH(launch_forward, a, stream);
}
template <int DT, int V>
cudaError_t backward_v(const NormBackArgs& a, uint32_t* ctas, cudaStream_t stream) {
  const uint32_t width = a.width;
  return GD_BY_WIDTH(launch_backward, a, ctas, stream);
}
#undef GD_BY_WIDTH

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
      const cudaError_t e = launch_dependent(norm_long_columns_kernel<DT>, dim3(across, *ctas), dim3(kLongColumnThreads), 0, stream, a);
      if (e != cudaSuccess) return e;
      note_launches(1);
    }
    return a.dx ? launch_dependent(norm_back_long_kernel<DT>, dim3(std::min(a.rows, 2u * (uint32_t)sm_count())), dim3(kMostThreads), 0, stream, a) : cudaSuccess;
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
    ProfileScope ps(stream, PT_NORM_BACK);
    const cudaError_t e = g->dtype == GD_DTYPE_FP32   ? backward_t<GD_DTYPE_FP32>(a, &ctas, stream)
                          : g->dtype == GD_DTYPE_BF16 ? backward_t<GD_DTYPE_BF16>(a, &ctas, stream)
                                                      : backward_t<GD_DTYPE_FP16>(a, &ctas, stream);
    if (e != cudaSuccess) return GD_ERR_CUDA;
    note_launches(1);
  }
  if (sums) {
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
