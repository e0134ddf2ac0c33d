// A gated linear recurrence over packed sequences (gd_recurrence_forward, gd_recurrence_backward).
//
// h[t] = f[t] h[t-1] + s[t] v[t] with f = sigmoid(gate), s = 1 - f is a composition of affine maps, column by column: rows t0 .. t1 take a state h to
// A h + B, and maps compose.  A CTA takes a slab of columns of one sequence, kTileRows rows at a time: each warp makes the map of its kRows rows
// in registers, the warps' maps meet in shared memory, and from the state that enters the tile every warp goes through its rows again, still
// in registers, and writes them.  So gate and value are read once and y is written once, whatever the length: bound by the bytes.  The next tile's
// rows are asked for before this one's are worked on.  Where sequences and slabs alone would leave SMs idle, a cluster of 2 .. 8 CTAs takes
// neighbouring tiles of a sequence and exchanges their maps (sent and counted, as the cross-entropy does).
//
// Backwards dh runs through the same maps from the other end: with C the map's constant, the gradient that leaves rows t0 .. t1 towards the past is
// A (what came in) + C.  The states h[t-1] that dgate needs are made again from the marks, the states before every kTileRows-th row of a sequence
// which the forward call keeps in fp32: y is rounded and would not do where h[t-1] and value nearly agree.
//
// Sequences of few rows (kShortRows on average, the single step among them): a thread takes a sequence's columns through all its rows.
#include <algorithm>
#include <cstring>

#include "gd_layers.cuh"
#include "gd_mma.cuh"

namespace gd {
namespace {

constexpr uint32_t kWarps = 8, kRows = 8, kTileRows = kWarps * kRows;      // kTileRows is part of the marks' layout
constexpr uint32_t kShortRows = 24;
constexpr uint32_t kMostCluster = 8;

struct Spans {
  const void* offsets;
  uint32_t bits, rows, sequences;
  // first row of a sequence and how many it has; offsets that make no sense are cut to what does
  __device__ __forceinline__ void of(uint32_t s, uint32_t* first, uint32_t* count) const {
    if (!offsets) {
      const uint32_t per = rows / sequences;
      *first = s * per, *count = per;
      return;
    }
    int64_t b, e;
    if (bits == 64) b = static_cast<const int64_t*>(offsets)[s], e = static_cast<const int64_t*>(offsets)[s + 1];
    else b = static_cast<const int32_t*>(offsets)[s], e = static_cast<const int32_t*>(offsets)[s + 1];
    b = min(max(b, (int64_t)0), (int64_t)rows);
    e = min(max(e, b), (int64_t)rows);
    *first = (uint32_t)b, *count = (uint32_t)(e - b);
  }
};
struct ScanArgs {
  Spans spans;
  const void* gate;
  const void* value;
  void* y;
  uint64_t ld_gate, ld_value, ld_y;
  const float* h0;
  float* h_last;
  float* marks;
  uint32_t width, slabs;
  uint64_t items;              // (sequence, slab)
};
struct ScanBackArgs {
  Spans spans;
  const void* dy;
  const void* gate;
  const void* value;
  const float* marks;
  void* dgate;
  void* dvalue;
  uint64_t ld_dy, ld_gate, ld_value, ld_dgate, ld_dvalue;
  const float* dh_last;
  float* dh0;
  uint32_t width, slabs;
  uint64_t items;
};
// the row of marks that holds the state before row 0 of a sequence
__device__ __forceinline__ uint64_t first_mark(uint32_t sequence, uint32_t first_row) { return (uint64_t)first_row / kTileRows + sequence; }

// f = 1 / (1 + exp(-g)) and s = 1 - f, each to its own relative accuracy
template <int DT>
__device__ __forceinline__ void gate_of(float g, float* f, float* s) {
  const float e = DT == GD_DTYPE_FP32 ? expf(-fabsf(g)) : __expf(-fabsf(g));
  const float big = __fdividef(1.f, 1.f + e), small = e * big;
  *f = g < 0.f ? small : big;      // (a NaN stays one)
  *s = g < 0.f ? big : small;
}

// ---------------------------------------------------------------- exchange of a cluster's maps
// Two places in turn for the pairs of all CTAs, each counted on an mbarrier of its own.
template <int V>
struct Exchange {
  float2 pair[2][kMostCluster][32 * V];
  uint64_t full[2];
};
template <int V>
__device__ __forceinline__ void exchange_begin(Exchange<V>& x, uint32_t cluster) {
  if (threadIdx.x == 0) {
    for (int b = 0; b < 2; ++b) {
      mbar_init(&x.full[b], 1u);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      mbar_arrive_expect_tx(&x.full[b], cluster * 32u * V * 8u);
    }
  }
  __syncthreads();
  cluster_arrive();
  cluster_wait();
}
// Sends this CTA's (a, b) to all and waits for everybody's.  Warp w sends to CTA w; all threads hold the same values for their lane's columns.
template <int V>
__device__ __forceinline__ bool exchange(Exchange<V>& x, uint32_t cluster, uint32_t rank, uint32_t round, const float (&a)[V], const float (&b)[V]) {
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, at = round & 1u;
  if (warp < cluster) {
    const uint32_t full = peer_address(smem_u32(&x.full[at]), warp);
#pragma unroll
    for (int i = 0; i < V; ++i) send_peer2(peer_address(smem_u32(&x.pair[at][rank][lane * V + i]), warp), make_float2(a[i], b[i]), full);
  }
  const int never = 0;
  return mbar_wait(&x.full[at], (round >> 1) & 1u, &never);
}
// after all threads are past the wait of `round`, and before they send for round + 2
template <int V>
__device__ __forceinline__ void exchange_again(Exchange<V>& x, uint32_t cluster, uint32_t round) {
  if (threadIdx.x == 0) mbar_arrive_expect_tx(&x.full[round & 1u], cluster * 32u * V * 8u);
}

// ---------------------------------------------------------------- forward
template <int DT, int V, bool CLUSTER>
__global__ void __launch_bounds__(kWarps * 32) scan_kernel(const __grid_constant__ ScanArgs a, uint32_t cluster) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  __shared__ float2 s_map[2][kWarps][32 * V];
  __shared__ Exchange<CLUSTER ? V : 1> s_x;
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, rank = CLUSTER ? cluster_rank() : 0u;
  if constexpr (CLUSTER) exchange_begin(s_x, cluster);
  pdl_wait();
  pdl_trigger();
  uint32_t turn = 0, round = 0;
  const uint64_t stride = gridDim.x / cluster;
  for (uint64_t item = blockIdx.x / cluster; item < a.items; item += stride) {
    const uint32_t seq = (uint32_t)(item / a.slabs), c = ((uint32_t)(item % a.slabs) * 32u + lane) * V;
    uint32_t first, count;
    a.spans.of(seq, &first, &count);
    const bool in = c < a.width;
    const T* gate = static_cast<const T*>(a.gate) + (uint64_t)first * a.ld_gate + c;
    const T* value = static_cast<const T*>(a.value) + (uint64_t)first * a.ld_value + c;
    T* y = static_cast<T*>(a.y) + (uint64_t)first * a.ld_y + c;
    const uint64_t mark0 = first_mark(seq, first);
    float h[V];
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = in && a.h0 ? a.h0[(uint64_t)seq * a.width + c + i] : 0.f;
    const uint32_t tiles = (count + kTileRows - 1) / kTileRows;
    typename P::Raw next_g[kRows], next_v[kRows];
    const auto ask = [&](uint32_t tile) {
      const uint32_t r0 = tile * kTileRows + warp * kRows;
#pragma unroll
      for (uint32_t k = 0; k < kRows; ++k) {
        const bool there = in && tile < tiles && r0 + k < count;
        next_g[k] = there ? P::load(gate + (uint64_t)(r0 + k) * a.ld_gate) : P::none();
        next_v[k] = there ? P::load(value + (uint64_t)(r0 + k) * a.ld_value) : P::none();
      }
    };
    ask(rank);
    for (uint32_t tile = rank; tile - rank < tiles; tile += cluster) {
      const uint32_t r0 = tile * kTileRows + warp * kRows, rows = tile < tiles && r0 < count ? min(kRows, count - r0) : 0u;
      float f[kRows][V], sv[kRows][V], A[V], B[V];
#pragma unroll
      for (int i = 0; i < V; ++i) A[i] = 1.f, B[i] = 0.f;
#pragma unroll
      for (uint32_t k = 0; k < kRows; ++k) {
        float g[V], v[V];
        P::widen(next_g[k], g);
        P::widen(next_v[k], v);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float s;
          gate_of<DT>(g[i], &f[k][i], &s);
          sv[k][i] = s * v[i];
          if (k >= rows) f[k][i] = 1.f, sv[k][i] = 0.f;
          A[i] *= f[k][i];
          B[i] = fmaf(f[k][i], B[i], sv[k][i]);
        }
      }
      ask(tile + cluster);
      float2(*map)[32 * V] = s_map[turn & 1u];
      ++turn;
#pragma unroll
      for (int i = 0; i < V; ++i) map[warp][lane * V + i] = make_float2(A[i], B[i]);
      __syncthreads();
      if constexpr (CLUSTER) {
        // the tile's map; from the others' the state that enters this tile, and the one behind the cluster's tiles
#pragma unroll
        for (int i = 0; i < V; ++i) {
          A[i] = 1.f, B[i] = 0.f;
#pragma unroll
          for (uint32_t w = 0; w < kWarps; ++w) {
            const float2 m = map[w][lane * V + i];
            A[i] *= m.x, B[i] = fmaf(m.x, B[i], m.y);
          }
        }
        const bool good = exchange(s_x, cluster, rank, round, A, B);
        float after[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float e = good ? h[i] : NAN, mine = e;
          for (uint32_t q = 0; q < cluster; ++q) {
            if (q == rank) mine = e;
            const float2 m = s_x.pair[round & 1u][q][lane * V + i];
            e = fmaf(m.x, e, m.y);
          }
          h[i] = mine, after[i] = e;
        }
        if (a.marks && in && tile < tiles && warp == 0) {
#pragma unroll
          for (int i = 0; i < V; ++i) a.marks[(mark0 + tile) * a.width + c + i] = h[i];
        }
#pragma unroll
        for (int i = 0; i < V; ++i) {
#pragma unroll
          for (uint32_t w = 0; w < kWarps; ++w) {
            const float2 m = map[w][lane * V + i];
            h[i] = w < warp ? fmaf(m.x, h[i], m.y) : h[i];
          }
        }
#pragma unroll
        for (uint32_t k = 0; k < kRows; ++k) {
#pragma unroll
          for (int i = 0; i < V; ++i) h[i] = fmaf(f[k][i], h[i], sv[k][i]);
          if (in && k < rows) P::store(y + (uint64_t)(r0 + k) * a.ld_y, P::narrow(h));
        }
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = after[i];
        exchange_again(s_x, cluster, round);
        ++round;
      } else {
        if (a.marks && in && warp == 0) {
#pragma unroll
          for (int i = 0; i < V; ++i) a.marks[(mark0 + tile) * a.width + c + i] = h[i];
        }
        float mine[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          mine[i] = h[i];
#pragma unroll
          for (uint32_t w = 0; w < kWarps; ++w) {
            if (w == warp) mine[i] = h[i];
            const float2 m = map[w][lane * V + i];
            h[i] = fmaf(m.x, h[i], m.y);
          }
        }
#pragma unroll
        for (uint32_t k = 0; k < kRows; ++k) {
#pragma unroll
          for (int i = 0; i < V; ++i) mine[i] = fmaf(f[k][i], mine[i], sv[k][i]);
          if (in && k < rows) P::store(y + (uint64_t)(r0 + k) * a.ld_y, P::narrow(mine));
        }
      }
    }
    // (h_last may be h0: written when all have read it)
    if constexpr (CLUSTER) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    if (a.h_last && in && warp == 0 && rank == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) a.h_last[(uint64_t)seq * a.width + c + i] = h[i];
    }
  }
  if constexpr (CLUSTER) {
    cluster_arrive();
    cluster_wait();
  }
}

// One thread per sequence and V columns.
constexpr uint32_t kShortThreads = 128, kShortAhead = 4;
template <int DT, int V>
__global__ void __launch_bounds__(kShortThreads) scan_short_kernel(const __grid_constant__ ScanArgs a) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  pdl_wait();
  pdl_trigger();
  const uint64_t stride = (uint64_t)gridDim.x * kShortThreads;
  for (uint64_t t = (uint64_t)blockIdx.x * kShortThreads + threadIdx.x; t < a.items; t += stride) {      // (slabs: pieces of a row)
    const uint32_t seq = (uint32_t)(t / a.slabs), c = (uint32_t)(t % a.slabs) * V;
    uint32_t first, count;
    a.spans.of(seq, &first, &count);
    const T* gate = static_cast<const T*>(a.gate) + (uint64_t)first * a.ld_gate + c;
    const T* value = static_cast<const T*>(a.value) + (uint64_t)first * a.ld_value + c;
    T* y = static_cast<T*>(a.y) + (uint64_t)first * a.ld_y + c;
    const uint64_t mark0 = first_mark(seq, first);
    float h[V];
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = a.h0 ? a.h0[(uint64_t)seq * a.width + c + i] : 0.f;
    for (uint32_t r = 0; r < count; r += kShortAhead) {
      if (a.marks && r % kTileRows == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) a.marks[(mark0 + r / kTileRows) * a.width + c + i] = h[i];
      }
      typename P::Raw g_raw[kShortAhead], v_raw[kShortAhead];
#pragma unroll
      for (uint32_t k = 0; k < kShortAhead; ++k) {
        if (r + k >= count) continue;
        g_raw[k] = P::load(gate + (uint64_t)(r + k) * a.ld_gate);
        v_raw[k] = P::load(value + (uint64_t)(r + k) * a.ld_value);
      }
#pragma unroll
      for (uint32_t k = 0; k < kShortAhead; ++k) {
        if (r + k >= count) continue;
        float g[V], v[V];
        P::widen(g_raw[k], g);
        P::widen(v_raw[k], v);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float f, s;
          gate_of<DT>(g[i], &f, &s);
          h[i] = fmaf(f, h[i], s * v[i]);
        }
        P::store(y + (uint64_t)(r + k) * a.ld_y, P::narrow(h));
      }
    }
    if (a.h_last) {
#pragma unroll
      for (int i = 0; i < V; ++i) a.h_last[(uint64_t)seq * a.width + c + i] = h[i];
    }
  }
}

// ---------------------------------------------------------------- backward
template <int DT, int V, bool CLUSTER>
__global__ void __launch_bounds__(kWarps * 32, 2) scan_back_kernel(const __grid_constant__ ScanBackArgs a, uint32_t cluster) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  __shared__ float2 s_map[2][kWarps][32 * V];       // (A, B): of the states
  __shared__ float s_back[2][kWarps][32 * V];       // C: of the gradient
  __shared__ Exchange<CLUSTER ? V : 1> s_x;
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, rank = CLUSTER ? cluster_rank() : 0u;
  if constexpr (CLUSTER) exchange_begin(s_x, cluster);
  pdl_wait();
  pdl_trigger();
  uint32_t turn = 0, round = 0;
  const uint64_t stride = gridDim.x / cluster;
  for (uint64_t item = blockIdx.x / cluster; item < a.items; item += stride) {
    const uint32_t seq = (uint32_t)(item / a.slabs), c = ((uint32_t)(item % a.slabs) * 32u + lane) * V;
    uint32_t first, count;
    a.spans.of(seq, &first, &count);
    const bool in = c < a.width;
    const T* gate = static_cast<const T*>(a.gate) + (uint64_t)first * a.ld_gate + c;
    const T* value = static_cast<const T*>(a.value) + (uint64_t)first * a.ld_value + c;
    const T* dy = static_cast<const T*>(a.dy) + (uint64_t)first * a.ld_dy + c;
    T* dgate = static_cast<T*>(a.dgate) + (uint64_t)first * a.ld_dgate + c;
    T* dvalue = static_cast<T*>(a.dvalue) + (uint64_t)first * a.ld_dvalue + c;
    const float* marks = a.marks + first_mark(seq, first) * a.width + c;
    float carry[V];                                  // f[t+1] dh[t+1] of the row behind the tile
#pragma unroll
    for (int i = 0; i < V; ++i) carry[i] = in && a.dh_last ? a.dh_last[(uint64_t)seq * a.width + c + i] : 0.f;
    const uint32_t tiles = (count + kTileRows - 1) / kTileRows, sets = (tiles + cluster - 1) / cluster;
    typename P::Raw next_g[kRows], next_v[kRows], next_d[kRows];
    float next_h[V];
    const auto ask = [&](uint32_t set) {             // of the set-th group of tiles, counted from 1
      const uint32_t tile = (set - 1) * cluster + rank, r0 = tile * kTileRows + warp * kRows;
#pragma unroll
      for (uint32_t k = 0; k < kRows; ++k) {
        const bool there = in && set && tile < tiles && r0 + k < count;
        next_g[k] = there ? P::load(gate + (uint64_t)(r0 + k) * a.ld_gate) : P::none();
        next_v[k] = there ? P::load(value + (uint64_t)(r0 + k) * a.ld_value) : P::none();
        next_d[k] = there ? P::load(dy + (uint64_t)(r0 + k) * a.ld_dy) : P::none();
      }
#pragma unroll
      for (int i = 0; i < V; ++i) next_h[i] = in && set && tile < tiles ? marks[(uint64_t)tile * a.width + i] : 0.f;
    };
    ask(sets);
    for (uint32_t set = sets; set > 0; --set) {
      const uint32_t tile = (set - 1) * cluster + rank, r0 = tile * kTileRows + warp * kRows;
      const uint32_t rows = tile < tiles && r0 < count ? min(kRows, count - r0) : 0u;
      float f[kRows][V], s[kRows][V], v[kRows][V], A[V], B[V], C[V], h[V];
      typename P::Raw d_raw[kRows];
#pragma unroll
      for (int i = 0; i < V; ++i) A[i] = 1.f, B[i] = 0.f, C[i] = 0.f, h[i] = next_h[i];
#pragma unroll
      for (uint32_t k = 0; k < kRows; ++k) {
        float g[V];
        P::widen(next_g[k], g);
        P::widen(next_v[k], v[k]);
        d_raw[k] = next_d[k];
#pragma unroll
        for (int i = 0; i < V; ++i) {
          gate_of<DT>(g[i], &f[k][i], &s[k][i]);
          if (k >= rows) f[k][i] = 1.f, s[k][i] = 0.f;
          A[i] *= f[k][i];
          B[i] = fmaf(f[k][i], B[i], s[k][i] * v[k][i]);
        }
      }
#pragma unroll
      for (uint32_t k = kRows; k-- > 0;) {
        float d[V];
        P::widen(d_raw[k], d);
#pragma unroll
        for (int i = 0; i < V; ++i) C[i] = f[k][i] * (d[i] + C[i]);
      }
      ask(set - 1);
      float2(*map)[32 * V] = s_map[turn & 1u];
      float(*back)[32 * V] = s_back[turn & 1u];
      ++turn;
#pragma unroll
      for (int i = 0; i < V; ++i) map[warp][lane * V + i] = make_float2(A[i], B[i]), back[warp][lane * V + i] = C[i];
      __syncthreads();
      float behind[V];                               // what reaches the tile's last row
      if constexpr (CLUSTER) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          A[i] = 1.f, C[i] = 0.f;
#pragma unroll
          for (uint32_t w = kWarps; w-- > 0;) {
            const float m = map[w][lane * V + i].x;
            A[i] *= m, C[i] = fmaf(m, C[i], back[w][lane * V + i]);
          }
        }
        const bool good = exchange(s_x, cluster, rank, round, A, C);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float e = good ? carry[i] : NAN;
          behind[i] = e;
          for (uint32_t q = cluster; q-- > 0;) {
            if (q == rank) behind[i] = e;
            const float2 m = s_x.pair[round & 1u][q][lane * V + i];
            e = fmaf(m.x, e, m.y);
          }
          carry[i] = e;
        }
        exchange_again(s_x, cluster, round);
        ++round;
      } else {
#pragma unroll
        for (int i = 0; i < V; ++i) behind[i] = carry[i];
      }
      float g[V];
#pragma unroll
      for (int i = 0; i < V; ++i) {
        float e = behind[i];
        g[i] = e;
#pragma unroll
        for (uint32_t w = kWarps; w-- > 0;) {
          if (w == warp) g[i] = e;
          e = fmaf(map[w][lane * V + i].x, e, back[w][lane * V + i]);
        }
        if (!CLUSTER) carry[i] = e;
#pragma unroll
        for (uint32_t w = 0; w < kWarps; ++w) {
          const float2 m = map[w][lane * V + i];
          h[i] = w < warp ? fmaf(m.x, h[i], m.y) : h[i];
        }
      }
#pragma unroll
      for (uint32_t k = 0; k < kRows; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float before = h[i];
          h[i] = fmaf(f[k][i], h[i], s[k][i] * v[k][i]);
          v[k][i] = before - v[k][i];
        }
      }
#pragma unroll
      for (uint32_t k = kRows; k-- > 0;) {
        float d[V], dg[V], dv[V];
        P::widen(d_raw[k], d);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float dh = d[i] + g[i];
          dv[i] = s[k][i] * dh;
          g[i] = f[k][i] * dh;
          dg[i] = dv[i] * v[k][i] * f[k][i];
        }
        if (in && k < rows) {
          P::store(dgate + (uint64_t)(r0 + k) * a.ld_dgate, P::narrow(dg));
          P::store(dvalue + (uint64_t)(r0 + k) * a.ld_dvalue, P::narrow(dv));
        }
      }
    }
    if constexpr (CLUSTER) {
      cluster_arrive();
      cluster_wait();
    } else {
      __syncthreads();
    }
    if (a.dh0 && in && warp == 0 && rank == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) a.dh0[(uint64_t)seq * a.width + c + i] = carry[i];
    }
  }
  if constexpr (CLUSTER) {
    cluster_arrive();
    cluster_wait();
  }
}

// One thread per sequence and V columns: kShortAhead rows at a time from the last, their states made from the nearest mark.
template <int DT, int V>
__global__ void __launch_bounds__(kShortThreads) scan_back_short_kernel(const __grid_constant__ ScanBackArgs a) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  pdl_wait();
  pdl_trigger();
  const uint64_t stride = (uint64_t)gridDim.x * kShortThreads;
  for (uint64_t t = (uint64_t)blockIdx.x * kShortThreads + threadIdx.x; t < a.items; t += stride) {
    const uint32_t seq = (uint32_t)(t / a.slabs), c = (uint32_t)(t % a.slabs) * V;
    uint32_t first, count;
    a.spans.of(seq, &first, &count);
    const T* gate = static_cast<const T*>(a.gate) + (uint64_t)first * a.ld_gate + c;
    const T* value = static_cast<const T*>(a.value) + (uint64_t)first * a.ld_value + c;
    const T* dy = static_cast<const T*>(a.dy) + (uint64_t)first * a.ld_dy + c;
    T* dgate = static_cast<T*>(a.dgate) + (uint64_t)first * a.ld_dgate + c;
    T* dvalue = static_cast<T*>(a.dvalue) + (uint64_t)first * a.ld_dvalue + c;
    const float* marks = a.marks + first_mark(seq, first) * a.width + c;
    float g[V];
#pragma unroll
    for (int i = 0; i < V; ++i) g[i] = a.dh_last ? a.dh_last[(uint64_t)seq * a.width + c + i] : 0.f;
    for (uint32_t end = count; end > 0;) {
      const uint32_t r0 = (end - 1) / kShortAhead * kShortAhead, rows = end - r0;
      float h[V], f[kShortAhead][V], s[kShortAhead][V], v[kShortAhead][V];
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = marks[(uint64_t)(r0 / kTileRows) * a.width + i];
      // the state before r0 (a sequence this long among short ones goes through its rows several times)
      for (uint32_t r = r0 / kTileRows * kTileRows; r < r0; ++r) {
        float x[V], w[V];
        P::widen(P::load_kept(gate + (uint64_t)r * a.ld_gate), x);
        P::widen(P::load_kept(value + (uint64_t)r * a.ld_value), w);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          float p, q;
          gate_of<DT>(x[i], &p, &q);
          h[i] = fmaf(p, h[i], q * w[i]);
        }
      }
      typename P::Raw d_raw[kShortAhead];
#pragma unroll
      for (uint32_t k = 0; k < kShortAhead; ++k) {
        float x[V];
        if (k >= rows) continue;
        d_raw[k] = P::load(dy + (uint64_t)(r0 + k) * a.ld_dy);
        P::widen(P::load(gate + (uint64_t)(r0 + k) * a.ld_gate), x);
        P::widen(P::load(value + (uint64_t)(r0 + k) * a.ld_value), v[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          gate_of<DT>(x[i], &f[k][i], &s[k][i]);
          const float before = h[i];
          h[i] = fmaf(f[k][i], h[i], s[k][i] * v[k][i]);
          v[k][i] = before - v[k][i];
        }
      }
#pragma unroll
      for (uint32_t k = kShortAhead; k-- > 0;) {
        if (k >= rows) continue;
        float d[V], dg[V], dv[V];
        P::widen(d_raw[k], d);
#pragma unroll
        for (int i = 0; i < V; ++i) {
          const float dh = d[i] + g[i];
          dv[i] = s[k][i] * dh;
          g[i] = f[k][i] * dh;
          dg[i] = dv[i] * v[k][i] * f[k][i];
        }
        P::store(dgate + (uint64_t)(r0 + k) * a.ld_dgate, P::narrow(dg));
        P::store(dvalue + (uint64_t)(r0 + k) * a.ld_dvalue, P::narrow(dv));
      }
      end = r0;
    }
    if (a.dh0) {
#pragma unroll
      for (int i = 0; i < V; ++i) a.dh0[(uint64_t)seq * a.width + c + i] = g[i];
    }
  }
}

// ---------------------------------------------------------------- host side
template <typename Args>
cudaError_t launch_clusters(void (*kernel)(Args, uint32_t), const Args& a, uint32_t cluster, cudaStream_t stream) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)std::min<uint64_t>(a.items, 1u << 24) * cluster);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, cluster);
}
// CTAs per sequence and slab: more while SMs would be idle and every CTA has two tiles or more
uint32_t choose_cluster(uint64_t items, const Spans& s) {
  uint32_t cluster = 1;
  while (cluster < kMostCluster && items * cluster * 2 <= 2ull * sm_count() && s.rows / s.sequences >= 4ull * cluster * kTileRows) cluster *= 2;
  return cluster;
}
template <int DT, int V>
cudaError_t launch_forward(ScanArgs a, cudaStream_t stream) {
  if (a.spans.rows / a.spans.sequences < kShortRows) {
    a.slabs = a.width / V;
    a.items = (uint64_t)a.spans.sequences * a.slabs;
    const uint64_t ctas = std::min<uint64_t>((a.items + kShortThreads - 1) / kShortThreads, 1u << 24);
    return launch_dependent(scan_short_kernel<DT, V>, dim3((uint32_t)ctas), dim3(kShortThreads), 0, stream, a);
  }
  a.slabs = (a.width + 32 * V - 1) / (32 * V);
  a.items = (uint64_t)a.spans.sequences * a.slabs;
  const uint32_t cluster = choose_cluster(a.items, a.spans);
  return launch_clusters<ScanArgs>(cluster > 1 ? scan_kernel<DT, V, true> : scan_kernel<DT, V, false>, a, cluster, stream);
}
template <int DT, int V>
cudaError_t launch_backward(ScanBackArgs a, cudaStream_t stream) {
  if (a.spans.rows / a.spans.sequences < kShortRows) {
    a.slabs = a.width / V;
    a.items = (uint64_t)a.spans.sequences * a.slabs;
    const uint64_t ctas = std::min<uint64_t>((a.items + kShortThreads - 1) / kShortThreads, 1u << 24);
    return launch_dependent(scan_back_short_kernel<DT, V>, dim3((uint32_t)ctas), dim3(kShortThreads), 0, stream, a);
  }
  a.slabs = (a.width + 32 * V - 1) / (32 * V);
  a.items = (uint64_t)a.spans.sequences * a.slabs;
  const uint32_t cluster = choose_cluster(a.items, a.spans);
  return launch_clusters<ScanBackArgs>(cluster > 1 ? scan_back_kernel<DT, V, true> : scan_back_kernel<DT, V, false>, a, cluster, stream);
}

int check_shape(uint64_t rows, uint64_t sequences, uint64_t width, int dtype, const void* offsets, int offset_bits) {
  if (!is_dtype(dtype) || (offset_bits != 32 && offset_bits != 64)) return GD_ERR_INVALID_ARG;
  if (rows >> 31 || sequences >> 31 || width >> 31) return GD_ERR_TOO_LARGE;
  if (offsets ? !aligned_to(offsets, (size_t)offset_bits / 8) : sequences && rows % sequences) return GD_ERR_INVALID_ARG;
  if (!offsets && !sequences && rows) return GD_ERR_INVALID_ARG;
  return GD_OK;
}

int forward(const gd_recurrence_forward_args* g, cudaStream_t stream) {
  if (!g) return GD_ERR_INVALID_ARG;
  const int rc = check_shape(g->rows, g->sequences, g->width, g->dtype, g->offsets, g->offset_bits);
  if (rc != GD_OK) return rc;
  if (g->sequences == 0 || g->width == 0) return GD_OK;
  const size_t item = dtype_bytes(g->dtype);
  if (g->rows && (!good_matrix(g->gate, g->ld_gate, g->rows, g->width, item) || !good_matrix(g->value, g->ld_value, g->rows, g->width, item) ||
                  !good_matrix(g->y, g->ld_y, g->rows, g->width, item)))
    return GD_ERR_INVALID_ARG;
  if (!aligned_to(g->h0, 4) || !aligned_to(g->h_last, 4) || !aligned_to(g->marks, 4)) return GD_ERR_INVALID_ARG;
  ScanArgs a;
  std::memset(&a, 0, sizeof(a));
  a.spans = Spans{g->offsets, (uint32_t)g->offset_bits, (uint32_t)g->rows, (uint32_t)g->sequences};
  a.gate = g->gate, a.ld_gate = g->ld_gate;
  a.value = g->value, a.ld_value = g->ld_value;
  a.y = g->y, a.ld_y = g->ld_y;
  a.h0 = g->h0, a.h_last = g->h_last, a.marks = g->marks;
  a.width = (uint32_t)g->width;
  // two 16-bit columns a thread where rows take 4-byte accesses
  const auto pairs = [&](const void* p, uint64_t ld) { return in_pieces(p, ld, g->rows, g->width, item, 2); };
  const bool two = g->width % 2 == 0 && pairs(g->gate, g->ld_gate) && pairs(g->value, g->ld_value) && pairs(g->y, g->ld_y);
  ProfileScope ps(stream, PT_RECURRENCE);
  cudaError_t e;
  if (g->dtype == GD_DTYPE_FP32) e = launch_forward<GD_DTYPE_FP32, 1>(a, stream);
  else if (g->dtype == GD_DTYPE_BF16) e = two ? launch_forward<GD_DTYPE_BF16, 2>(a, stream) : launch_forward<GD_DTYPE_BF16, 1>(a, stream);
  else e = two ? launch_forward<GD_DTYPE_FP16, 2>(a, stream) : launch_forward<GD_DTYPE_FP16, 1>(a, stream);
  if (e != cudaSuccess) return GD_ERR_CUDA;
  note_launches(1);
  return GD_OK;
}

int backward(const gd_recurrence_backward_args* g, cudaStream_t stream) {
  if (!g) return GD_ERR_INVALID_ARG;
  const int rc = check_shape(g->rows, g->sequences, g->width, g->dtype, g->offsets, g->offset_bits);
  if (rc != GD_OK) return rc;
  if (g->sequences == 0 || g->width == 0) return GD_OK;
  const size_t item = dtype_bytes(g->dtype);
  const uint64_t rows = g->rows, width = g->width;
  if (rows && (!good_matrix(g->dy, g->ld_dy, rows, width, item) || !good_matrix(g->gate, g->ld_gate, rows, width, item) ||
               !good_matrix(g->value, g->ld_value, rows, width, item) || !good_matrix(g->dgate, g->ld_dgate, rows, width, item) ||
               !good_matrix(g->dvalue, g->ld_dvalue, rows, width, item) || !g->marks))
    return GD_ERR_INVALID_ARG;
  if (!aligned_to(g->dh_last, 4) || !aligned_to(g->dh0, 4) || !aligned_to(g->marks, 4)) return GD_ERR_INVALID_ARG;
  if (rows > 1 && ((g->dgate == g->gate && g->ld_dgate != g->ld_gate) || (g->dgate == g->dy && g->ld_dgate != g->ld_dy) ||
                   (g->dvalue == g->value && g->ld_dvalue != g->ld_value)))
    return GD_ERR_INVALID_ARG;
  ScanBackArgs a;
  std::memset(&a, 0, sizeof(a));
  a.spans = Spans{g->offsets, (uint32_t)g->offset_bits, (uint32_t)rows, (uint32_t)g->sequences};
  a.dy = g->dy, a.ld_dy = g->ld_dy;
  a.gate = g->gate, a.ld_gate = g->ld_gate;
  a.value = g->value, a.ld_value = g->ld_value;
  a.marks = g->marks;
  a.dgate = g->dgate, a.ld_dgate = g->ld_dgate;
  a.dvalue = g->dvalue, a.ld_dvalue = g->ld_dvalue;
  a.dh_last = g->dh_last, a.dh0 = g->dh0;
  a.width = (uint32_t)width;
  const auto pairs = [&](const void* p, uint64_t ld) { return in_pieces(p, ld, rows, width, item, 2); };
  const bool two = g->width % 2 == 0 && pairs(g->dy, g->ld_dy) && pairs(g->gate, g->ld_gate) && pairs(g->value, g->ld_value) && pairs(g->dgate, g->ld_dgate) && pairs(g->dvalue, g->ld_dvalue);
  ProfileScope ps(stream, PT_RECURRENCE_BACK);
  cudaError_t e;
  if (g->dtype == GD_DTYPE_FP32) e = launch_backward<GD_DTYPE_FP32, 1>(a, stream);
  else if (g->dtype == GD_DTYPE_BF16) e = two ? launch_backward<GD_DTYPE_BF16, 2>(a, stream) : launch_backward<GD_DTYPE_BF16, 1>(a, stream);
  else e = two ? launch_backward<GD_DTYPE_FP16, 2>(a, stream) : launch_backward<GD_DTYPE_FP16, 1>(a, stream);
  if (e != cudaSuccess) return GD_ERR_CUDA;
  note_launches(1);
  return GD_OK;
}

}  // namespace
}  // namespace gd

extern "C" {

int gd_recurrence_marks_rows(uint64_t rows, uint64_t sequences, uint64_t* rows_out) {
  if (!rows_out) return GD_ERR_INVALID_ARG;
  if (rows >> 31 || sequences >> 31) return GD_ERR_TOO_LARGE;
  *rows_out = rows / gd::kTileRows + sequences;
  return GD_OK;
}
int gd_recurrence_forward(const gd_recurrence_forward_args* a, void* stream) { return gd::forward(a, (cudaStream_t)stream); }
int gd_recurrence_backward(const gd_recurrence_backward_args* a, void* stream) { return gd::backward(a, (cudaStream_t)stream); }

}  // extern "C"
