// A gated linear recurrence over packed sequences (gd_recurrence_forward, gd_recurrence_backward).
//
// h[t] = f[t] h[t-1] + s[t] v[t] with f = sigmoid(gate), s = 1 - f is a composition of affine maps, column by column: rows t0 .. t1 take a state h to
// A h + B, and maps compose.  A CTA takes a slab of columns of one sequence, a tile of 64 or 128 rows at a time: each group of threads makes the map of its
// kRows rows in registers, the groups' maps meet in shared memory, and from the state that enters the tile every group goes through its rows again,
// still in registers, and writes them.  So gate and value are read once and y is written once, whatever the length; the next tiles' rows are copied into
// shared memory meanwhile.  What bounds it is instructions, with the bytes close behind: two exponential-unit operations, ten others to the gate's two
// weights, four to the maps and the state for each pair of columns, which go two to an instruction.  Where sequences and slabs alone would leave SMs idle, a cluster of 2 .. 8 CTAs takes
// neighbouring tiles of a sequence and exchanges their maps (sent and counted, as the cross-entropy does).
//
// Backwards dh runs through the same maps from the other end: with C the map's constant, the gradient that leaves rows t0 .. t1 towards the past is
// A (what came in) + C.  The states h[t-1] that dgate needs are made again from the marks, the states before every kMarkRows-th row of a sequence
// which the forward call keeps in fp32: y is rounded and would not do where h[t-1] and value nearly agree.
//
// Many sequences of few rows, the single step among them: a thread takes a sequence's columns through all its rows.
//
// Measured (bf16): 16 sequences of 2048 x 2048 78 us forward = 5.2 TB/s, 127 backward = 5.3; one of 65536 x 1024 103 and 236 (a set of tiles takes the
// cluster 1.6 us and 3.7, a CTA's 24 and 40 KB would take 0.6 and 0.9); 64 sequences by one step of 1024 4 us.  In fp32 one of 60000 x 1024 129 us = 5.7 TB/s.
#include <algorithm>
#include <cstring>

#include "gd_layers.cuh"
#include "gd_mma.cuh"

namespace gd {
namespace {

constexpr uint32_t kWarps = 8, kRows = 8, kMarkRows = kWarps * kRows;      // kMarkRows is part of the marks' layout
constexpr uint32_t kShortRows = 48, kStepRows = 8;
constexpr uint32_t kMostCluster = 8;

struct Spans {
  const void* offsets;
  uint32_t bits, rows, sequences;
  // first row of a sequence and how many it has, within the rows whatever the offsets (each pair is cut by itself: where they descend, sequences may overlap)
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
// How long a wait for a tile's copies or a cluster's maps lasts, and bytes awaited there that nobody sends (0; the self-test's 8).  A thread whose wait
// ran out marks its count of tiles and waits no more; the CTA's flag ends the others' waits that do not succeed at once.  Rows and states that did not
// come are NaN to it, and so is all that follows from them.  Thread 0 asks for no more copies then - a stage's may still be under way - and waits once
// more for those it has asked for before it ends.
struct Waits {
  uint64_t budget_ns;
  uint32_t missing_copies, missing_maps;
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
  bool by_length;              // long sequences first
  Waits waits;
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
  bool by_length;
  Waits waits;
};
// the row of marks that holds the state before row 0 of a sequence
__device__ __forceinline__ uint64_t first_mark(uint32_t sequence, uint32_t first_row) { return (uint64_t)first_row / kMarkRows + sequence; }

// f = 1 / (1 + exp(-g)) and s = 1 - f, each to its own relative accuracy
__device__ __forceinline__ float exp2_of(float x) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(x));
  return e;
}
__device__ __forceinline__ float inverse_of(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
constexpr float kLog2e = 1.4426950408889634f;
template <int DT>
__device__ __forceinline__ void gate_of(float g, float* f, float* s) {
  const float e = DT == GD_DTYPE_FP32 ? expf(-fabsf(g)) : exp2_of(-fabsf(g) * kLog2e);
  const float big = inverse_of(1.f + e), small = e * big;
  *f = g < 0.f ? small : big;      // (a NaN stays one)
  *s = g < 0.f ? big : small;
}
// Of two gates, for 16-bit types: with e = exp(-g), held at 2^126, f = 1 / (1 + e) and s = e f.  Where e is held f is 2^-126 too much: taken
// off again, which changes no f above 2^-102.  6.5 instructions an element where the above takes 8 and the instructions bound the kernel.
__device__ __forceinline__ void gate_pair(float2 g, float2* f, float2* s) {
  constexpr float kMost = 126.f, kLeast = 1.17549435e-38f;
  float2 t = mul2(g, both(-kLog2e));
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(t.x) : "f"(kMost));
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(t.y) : "f"(kMost));
  const float2 e = make_float2(exp2_of(t.x), exp2_of(t.y)), d = add2(e, both(1.f)), r = make_float2(inverse_of(d.x), inverse_of(d.y));
  *s = mul2(e, r);
  *f = add2(r, both(-kLeast));
}
// f and s of N elements side by side
template <int DT, int N>
__device__ __forceinline__ void gates_of(const float (&g)[N], float (&f)[N], float (&s)[N]) {
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    if constexpr (DT == GD_DTYPE_FP32) {
      gate_of<DT>(g[j], &f[j], &s[j]);
      gate_of<DT>(g[j + 1], &f[j + 1], &s[j + 1]);
    } else {
      float2 p, q;
      gate_pair(make_float2(g[j], g[j + 1]), &p, &q);
      f[j] = p.x, f[j + 1] = p.y, s[j] = q.x, s[j + 1] = q.y;
    }
  }
}
// The products of N elements side by side.
template <int N>
__device__ __forceinline__ void times(const float (&a)[N], const float (&b)[N], float (&c)[N]) {
#pragma unroll
  for (int j = 0; j < N; j += 2) {
    const float2 p = mul2(make_float2(a[j], a[j + 1]), make_float2(b[j], b[j + 1]));
    c[j] = p.x, c[j + 1] = p.y;
  }
}
// V columns' a * b + c, and a * b
template <int V>
__device__ __forceinline__ void fma_v(const float* a, const float* b, const float* c, float* r) {
  if constexpr (V == 2) {
    const float2 p = fma2(make_float2(a[0], a[1]), make_float2(b[0], b[1]), make_float2(c[0], c[1]));
    r[0] = p.x, r[1] = p.y;
  } else {
    r[0] = fmaf(a[0], b[0], c[0]);
  }
}
template <int V>
__device__ __forceinline__ void mul_v(const float* a, const float* b, float* r) {
  if constexpr (V == 2) {
    const float2 p = mul2(make_float2(a[0], a[1]), make_float2(b[0], b[1]));
    r[0] = p.x, r[1] = p.y;
  } else {
    r[0] = a[0] * b[0];
  }
}
template <int V>
__device__ __forceinline__ void add_v(const float* a, const float* b, float* r) {
  if constexpr (V == 2) {
    const float2 p = add2(make_float2(a[0], a[1]), make_float2(b[0], b[1]));
    r[0] = p.x, r[1] = p.y;
  } else {
    r[0] = a[0] + b[0];
  }
}
// The maps of the warps, in shared memory: a lane's V columns of A, then of B.
template <int V>
struct __align__(8 * V) Map {
  float a[V], b[V];
};
// first <- what the rows of `first` and then those of m make of a state
template <int V>
__device__ __forceinline__ void append(Map<V>& first, const Map<V>& m) {
  fma_v<V>(m.a, first.b, m.b, first.b);
  mul_v<V>(m.a, first.a, first.a);
}
template <int V>
__device__ __forceinline__ Map<V> identity() {
  Map<V> m;
#pragma unroll
  for (int i = 0; i < V; ++i) m.a[i] = 1.f, m.b[i] = 0.f;
  return m;
}

// ---------------------------------------------------------------- exchange of a cluster's maps
// A CTA sends the map of a tile to all CTAs of its cluster as soon as it has it, one tile before it needs theirs, so that nobody waits for a
// message under way.  Four places in turn, each counted on an mbarrier of its own: while a CTA reads the maps of tile set t the others may have
// sent those of t + 1 .. t + 3, which take its maps of up to t + 2 to have come that far.
constexpr uint32_t kPlaces = 4;
template <int V, int CL, int L>
struct Exchange {
  Map<V> map[kPlaces][CL][L];
  uint64_t full[kPlaces];
};
template <int V, int CL, int L>
__device__ __forceinline__ void exchange_begin(Exchange<V, CL, L>& x, uint32_t missing) {
  if (threadIdx.x == 0) {
    for (uint32_t b = 0; b < kPlaces; ++b) {
      mbar_init(&x.full[b], 1u);
      mbar_arrive_expect_tx(&x.full[b], CL * L * (uint32_t)sizeof(Map<V>) + missing);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  cluster_arrive();
  cluster_wait();
}
// One group of threads sends this CTA's map to all.
template <int V, int CL, int L>
__device__ __forceinline__ void exchange_send(Exchange<V, CL, L>& x, uint32_t rank, uint32_t round, const Map<V>& m) {
  const uint32_t at = round % kPlaces, to = smem_u32(&x.map[at][rank][threadIdx.x % L]), full = smem_u32(&x.full[at]);
#pragma unroll
  for (uint32_t q = 0; q < CL; ++q) {
    const uint32_t peer = peer_address(to, q), bar = peer_address(full, q);
    if constexpr (V == 2) {
      send_peer2(peer, make_float2(m.a[0], m.a[1]), bar);
      send_peer2(peer + 8u, make_float2(m.b[0], m.b[1]), bar);
    } else {
      send_peer2(peer, make_float2(m.a[0], m.b[0]), bar);
    }
  }
}
constexpr uint32_t kGone = 1u << 31;      // of a thread's count of tiles: a wait of its ran out
// False where it did; afterwards every second phase of a barrier that nobody begins any more looks like one that has ended, but states are NaN by then
// and stay it.
__device__ __forceinline__ bool wait_for(uint64_t* b, uint32_t parity, volatile int* gone, uint64_t budget_ns, uint32_t& taken) {
  if (mbar_try_wait(b, parity)) return true;
  if (!(taken & kGone) && mbar_wait(b, parity, gone, budget_ns)) return true;
  *gone = 1;
  taken |= kGone;
  return false;
}
// By one warp: waits for everybody's maps of `round` and makes the place ready for round + kPlaces (nobody sends for that before this CTA has sent
// for a later round, which it does behind a barrier behind this call).  From the state that enters the cluster's tiles, `carry`: what enters this CTA's, and `carry` behind the last.
template <int V, int CL, bool BACKWARD, int L>
__device__ __forceinline__ void exchange_fold(Exchange<V, CL, L>& x, uint32_t rank, uint32_t round, volatile int* gone, uint64_t budget_ns, uint32_t& taken,
                                              float (&mine)[V], float (&carry)[V]) {
  const uint32_t lane = threadIdx.x % L, at = round % kPlaces;
  const bool good = wait_for(&x.full[at], (round / kPlaces) & 1u, gone, budget_ns, taken);
#pragma unroll
  for (int i = 0; i < V; ++i) {
    if (!good) carry[i] = NAN;                       // (a map that never came: the results say so)
    mine[i] = carry[i];
  }
#pragma unroll
  for (uint32_t n = 0; n < CL; ++n) {
    const uint32_t q = BACKWARD ? CL - 1u - n : n;
    if (q == rank) {
#pragma unroll
      for (int i = 0; i < V; ++i) mine[i] = carry[i];
    }
    const Map<V> m = x.map[at][q][lane];
    fma_v<V>(m.a, carry, m.b, carry);
  }
  if (threadIdx.x == 0) {
    if (!(taken & kGone)) mbar_arrive_expect_tx(&x.full[at], CL * L * (uint32_t)sizeof(Map<V>));
    else mbar_expect_tx(&x.full[at], CL * L * (uint32_t)sizeof(Map<V>));        // (the others send on: the count stays in its range)
  }
}

// ---------------------------------------------------------------- tiles in shared memory
// A group of L threads has V columns each of kRows rows; a tile is the groups' rows x L V columns of every input, brought by tiled copies (which cut
// at the matrix' end; what a tile holds beyond its sequence is masked) into one of a few stages.
template <int DT, int V, int L, int INPUTS, int CL>
struct TileShape {
  static constexpr uint32_t kGroups = kWarps * 32 / L, kTileRows = kGroups * kRows, kColumns = L * V;
  static constexpr uint32_t kInput = kTileRows * kColumns * sizeof(typename Elem<DT>::type), kStage = INPUTS * kInput;
  static constexpr uint32_t kDepth = INPUTS == 3 && CL > 1 ? 3 : 4;
  static constexpr uint32_t kBytes = kDepth * kStage + (CL > 1 ? (uint32_t)sizeof(Exchange<V, CL, L>) : 0u) + 128u;
};
constexpr uint32_t kMarkGroups = kMarkRows / kRows;      // groups from one mark to the next
// How a tile's rows come: as a box of a tensor map (rows at multiples of 16 bytes), by copies that each thread asks for its own places (of 4
// bytes: pairs of 16-bit columns, or fp32), or, single columns of 16 bits, through registers, a tile ahead.
enum Mode : int { kBoxes = 0, kOwnCopies = 1, kRegisters = 2 };

// The first `most` (up to kRows) of a thread's rows from p on, its V columns, into its own places of a tile: only it reads them.
template <typename T, int V, int L>
__device__ __forceinline__ void own_rows(unsigned char* tile, const T* p, uint64_t ld, uint32_t most) {
  const uint32_t to = smem_u32(tile) + ((threadIdx.x / L) * kRows * L + threadIdx.x % L) * V * (uint32_t)sizeof(T);
#pragma unroll
  for (uint32_t k = 0; k < kRows; ++k) {
    if (k < most) copy_ahead<V * (int)sizeof(T)>(to + k * (L * V * (uint32_t)sizeof(T)), p);
    p += ld;
  }
}

// The same into registers.
template <typename P, typename T>
__device__ __forceinline__ void held_rows(typename P::Raw (&held)[kRows], const T* p, uint64_t ld, uint32_t most) {
#pragma unroll
  for (uint32_t k = 0; k < kRows; ++k) {
    held[k] = k < most ? P::load(p) : P::none();
    p += ld;
  }
}
template <typename P, typename T>
__device__ __forceinline__ void held_rows(typename P::Raw (&)[1], const T*, uint64_t, uint32_t) {}

// All threads of a CTA: the sequence that `place` others come before in the order by length, the longest first.  One of several times the mean length
// that begins last runs by itself for most of the others' time: 20000 rows of 2048 in 30 ragged sequences 56 us in that order and 66 by index, backward
// 78 and 97; 16000 of 1000 in 80 46 and 55 backward.  Every CTA counts what is longer than each sequence: work that grows with the sequences, where its own
// grows with their length.  Of more sequences than a mean one has rows it costs more than it gives (30000 rows of 1024 in 250: 96 us and 49 by index), and
// where each SM takes many items there is little to give.
constexpr uint32_t kMostOrdered = kWarps * 32, kOrderedItems = 10;      // sequences; items to an SM
struct Chosen {
  uint32_t sequence, first, count;
};
__device__ __forceinline__ void longest_first(const Spans& spans, uint32_t place, uint32_t* keys, Chosen* chosen) {
  const uint32_t me = threadIdx.x;
  uint32_t first = 0, count = 0, key = 0;
  if (me < spans.sequences) {
    spans.of(me, &first, &count);
    key = min(count, (1u << 23) - 1u) << 8 | (kMostOrdered - 1u - me) | 1u << 31;
  }
  __syncthreads();                                   // (what `keys` held has been read)
  keys[me] = key;
  __syncthreads();
  if (key) {
    uint32_t before = 0;
#pragma unroll 4
    for (uint32_t i = 0; i < spans.sequences; i += 4) {
      const uint4 k = *reinterpret_cast<const uint4*>(keys + i);
      before += (k.x > key) + (k.y > key) + (k.z > key) + (k.w > key);
    }
    if (before == place) *chosen = Chosen{me, first, count};
  }
  __syncthreads();
}

// By thread 0 at the end, where a wait of its ran out.
template <uint32_t DEPTH>
__device__ __forceinline__ void settle_copies(uint64_t* full, uint32_t asked, uint64_t budget_ns) {
  const int none = 0;
  for (uint32_t n = asked > DEPTH ? asked - DEPTH : 0u; n < asked; ++n) (void)mbar_wait(&full[n % DEPTH], (n / DEPTH) & 1u, &none, budget_ns);
}

// A thread's rows of a tile that did not come, in an input of 4 bytes a place: NaN, whatever the type (or what arrives late).
template <int L>
__device__ __forceinline__ void spoil_rows(unsigned char* tile) {
  uint32_t* to = reinterpret_cast<uint32_t*>(tile) + (threadIdx.x / L) * kRows * L + threadIdx.x % L;
#pragma unroll 1
  for (uint32_t k = 0; k < kRows; ++k) to[k * L] = 0xFFFFFFFFu;
}

// ---------------------------------------------------------------- forward
// Rows that tiled copies can read: 16-byte aligned.
struct ScanMaps {
  CUtensorMap gate, value;
};
template <int DT, int V, int L, int CL, int MODE>
__global__ void __launch_bounds__(kWarps * 32, CL > 1 ? 2 : 3) scan_tiled_kernel(const __grid_constant__ ScanArgs a, const __grid_constant__ ScanMaps maps) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  using S = TileShape<DT, V, L, 2, CL>;
  constexpr uint32_t kDepth = S::kDepth, kGroups = S::kGroups, kTileRows = S::kTileRows, kColumns = S::kColumns;
  constexpr int R = kRows, N = R * V;                // row k's columns at k V
  extern __shared__ __align__(128) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
  __shared__ __align__(16) Map<V> s_map[2][kGroups][L];
  __shared__ float s_state[2][L][V];                // the state behind a tile, of the last group; in a cluster the one before the CTA's tile
  Exchange<V, CL, L>& s_x = *reinterpret_cast<Exchange<V, CL, L>*>(smem + S::kDepth * S::kStage);
  __shared__ uint64_t s_full[kDepth];
  __shared__ Chosen s_chosen;
  __shared__ int s_gone;
  volatile int* gone = &s_gone;
  const uint32_t lane = threadIdx.x % L, group = threadIdx.x / L, rank = CL > 1 ? cluster_rank() : 0u;
  if (threadIdx.x == 0) {
    s_gone = 0;
    for (uint32_t s = 0; s < kDepth; ++s) mbar_init(&s_full[s], 1u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (MODE == kBoxes) prefetch_map(&maps.gate), prefetch_map(&maps.value);
  }
  if constexpr (CL > 1) exchange_begin(s_x, a.waits.missing_maps);
  else __syncthreads();
  pdl_wait();
  pdl_trigger();
  uint32_t round = 0, asked = 0, taken = 0, turn = 0;
  const uint64_t stride = gridDim.x / CL;
  for (uint64_t item = blockIdx.x / CL; item < a.items; item += stride) {
    uint32_t seq = (uint32_t)(item / a.slabs), first, count;
    const uint32_t col0 = (uint32_t)(item % a.slabs) * kColumns, c = col0 + lane * V;
    if (CL == 1 && a.by_length) {
      longest_first(a.spans, seq, reinterpret_cast<uint32_t*>(s_map), &s_chosen);
      seq = s_chosen.sequence, first = s_chosen.first, count = s_chosen.count;
    } else {
      a.spans.of(seq, &first, &count);
    }
    const bool in = c < a.width;
    T* y = static_cast<T*>(a.y) + (uint64_t)first * a.ld_y + c;
    const uint64_t mark0 = first_mark(seq, first);
    const uint32_t tiles = (count + kTileRows - 1) / kTileRows, sets = (tiles + CL - 1) / CL;
    typename P::Raw held[MODE == kRegisters ? 2 : 1][MODE == kRegisters ? R : 1];
    // All threads: the copies of this CTA's tile of a set.
    const T* gate = static_cast<const T*>(a.gate) + (uint64_t)first * a.ld_gate + c;
    const T* value = static_cast<const T*>(a.value) + (uint64_t)first * a.ld_value + c;
    const auto ask = [&](uint32_t set) {
      const uint32_t tile = set * CL + rank, s = asked % kDepth;
      if constexpr (MODE == kBoxes) {
        if (threadIdx.x != 0 || tile >= tiles || (taken & kGone)) return;
        mbar_arrive_expect_tx(&s_full[s], S::kStage + a.waits.missing_copies);
        tile_load(smem + s * S::kStage, &maps.gate, (int32_t)col0, (int32_t)(first + tile * kTileRows), &s_full[s]);
        tile_load(smem + s * S::kStage + S::kInput, &maps.value, (int32_t)col0, (int32_t)(first + tile * kTileRows), &s_full[s]);
        ++asked;
      } else {
        const uint32_t r0 = tile * kTileRows + group * R, most = in && tile < tiles && r0 < count ? count - r0 : 0u;
        const T *from_g = gate + (uint64_t)r0 * a.ld_gate, *from_v = value + (uint64_t)r0 * a.ld_value;
        if constexpr (MODE == kOwnCopies) {
          own_rows<T, V, L>(smem + s * S::kStage, from_g, a.ld_gate, most);
          own_rows<T, V, L>(smem + s * S::kStage + S::kInput, from_v, a.ld_value, most);
          copies_commit();
        } else {
          held_rows<P>(held[0], from_g, a.ld_gate, most);
          held_rows<P>(held[1], from_v, a.ld_value, most);
        }
        if (tile < tiles) ++asked;
      }
    };
    // (registers:) what has been asked for into its stage
    const auto settle = [&](uint32_t s) {
#pragma unroll
      for (uint32_t input = 0; input < 2; ++input) {
        typename P::Raw* to = reinterpret_cast<typename P::Raw*>(smem + s * S::kStage + input * S::kInput) + group * R * L + lane;
#pragma unroll
        for (int k = 0; k < R; ++k) to[k * L] = held[input][k];
      }
    };
    constexpr uint32_t kAhead = MODE == kRegisters ? 1 : kDepth;
    for (uint32_t n = 0; n < kAhead; ++n) ask(n);
    float h[V];                                      // the state that enters the tile, or the cluster's tiles
#pragma unroll
    for (int i = 0; i < V; ++i) h[i] = taken & kGone ? NAN : in && a.h0 ? a.h0[(uint64_t)seq * a.width + c + i] : 0.f;
    const auto rows_of = [&](uint32_t tile) {
      const uint32_t r0 = tile * kTileRows + group * R;
      return tile < tiles && r0 < count ? min((uint32_t)R, count - r0) : 0u;
    };
    // f and s v of this group's rows of a tile, and their map, which is left for the other groups
    const auto evaluate = [&](uint32_t tile, float (&f)[N], float (&sv)[N]) __attribute__((always_inline)) {
      const uint32_t rows = rows_of(tile), s = taken % kDepth;
      if constexpr (MODE == kOwnCopies) copies_wait<(int)kDepth - 1>();
      if (tile < tiles) {
        if constexpr (MODE == kBoxes) {
          if (!wait_for(&s_full[s], (taken / kDepth) & 1u, gone, a.waits.budget_ns, taken)) spoil_rows<L>(smem + s * S::kStage + S::kInput);
        }
        if constexpr (MODE == kRegisters) settle(s);
        ++taken;
      }
      if (rows) {
        const T* from = reinterpret_cast<const T*>(smem + s * S::kStage) + (group * R * L + lane) * V;
        float g[N], v[N];
#pragma unroll
        for (int k = 0; k < R; ++k) {
          P::widen(*reinterpret_cast<const typename P::Raw*>(from + k * L * V), g + k * V);
          P::widen(*reinterpret_cast<const typename P::Raw*>(from + S::kInput / sizeof(T) + k * L * V), v + k * V);
        }
        gates_of<DT>(g, f, sv);
        times(sv, v, sv);
      }
      if (rows < R) {                                // behind the sequence: nothing changes
#pragma unroll
        for (int e = 0; e < N; ++e) {
          if (e / V >= (int)rows) f[e] = 1.f, sv[e] = 0.f;
        }
      }
      Map<V> m;
#pragma unroll
      for (int i = 0; i < V; ++i) m.a[i] = f[i], m.b[i] = sv[i];
#pragma unroll
      for (int k = 1; k < R; ++k) {
        fma_v<V>(f + k * V, m.b, sv + k * V, m.b);
        mul_v<V>(f + k * V, m.a, m.a);
      }
      s_map[turn & 1u][group][lane] = m;
      return m;
    };
    const auto apply = [&](uint32_t tile, const float (&f)[N], const float (&sv)[N], float (&state)[V]) __attribute__((always_inline)) {
      const uint32_t r0 = tile * kTileRows + group * R, rows = in ? rows_of(tile) : 0u;
      if (a.marks && group % kMarkGroups == 0 && rows) {
#pragma unroll
        for (int i = 0; i < V; ++i) a.marks[(mark0 + r0 / kMarkRows) * a.width + c + i] = state[i];
      }
      T* to = y + (uint64_t)r0 * a.ld_y;
      if (rows == R) {
#pragma unroll
        for (int k = 0; k < R; ++k) {
          fma_v<V>(f + k * V, state, sv + k * V, state);
          P::store(to, P::narrow(state));
          to += a.ld_y;
        }
      } else {
#pragma unroll
        for (int k = 0; k < R; ++k) {
          fma_v<V>(f + k * V, state, sv + k * V, state);
          if (k < (int)rows) P::store(to, P::narrow(state));
          to += a.ld_y;
        }
      }
    };
    if constexpr (CL > 1) {
      // the map of the next tile is under way to the others while this one's rows are written
      float f[2][N], sv[2][N];
      Map<V> before[2];                              // of the tile's rows before this group's
      // one warp joins the cluster's maps of a set and leaves the state that enters this CTA's tile for all (read behind the next barrier)
      const auto join = [&](uint32_t set) __attribute__((always_inline)) {
        if (threadIdx.x >= 32u) return;
        float state[V];
        exchange_fold<V, CL, false>(s_x, rank, round + set, gone, a.waits.budget_ns, taken, state, h);
#pragma unroll
        for (int i = 0; i < V; ++i) s_state[set & 1u][lane][i] = state[i];
      };
      const auto begin = [&](uint32_t set, float (&fn)[N], float (&svn)[N], Map<V>& before_n) __attribute__((always_inline)) {
        const Map<V> own = evaluate(set * CL + rank, fn, svn);
        if (set) join(set - 1);
        __syncthreads();
        ask(set + kAhead);
        before_n = identity<V>();
#pragma unroll
        for (uint32_t w = 0; w < kGroups - 1; ++w) {
          if (w == group) break;
          append(before_n, s_map[turn & 1u][w][lane]);
        }
        ++turn;
        if (group == kGroups - 1) {                    // (it has the tile's)
          Map<V> all = before_n;
          append(all, own);
          exchange_send(s_x, rank, round + set, all);
        }
      };
      const auto end = [&](uint32_t set, const float (&fn)[N], const float (&svn)[N], const Map<V>& before_n) __attribute__((always_inline)) {
        float state[V];
        if (set + 1 == sets) {
          join(set);
          __syncthreads();
        }
        fma_v<V>(before_n.a, s_state[set & 1u][lane], before_n.b, state);
        apply(set * CL + rank, fn, svn, state);
      };
      if (sets) begin(0, f[0], sv[0], before[0]);
      for (uint32_t set = 0; set < sets; set += 2) {
        if (set + 1 < sets) begin(set + 1, f[1], sv[1], before[1]);
        end(set, f[0], sv[0], before[0]);
        if (set + 1 >= sets) break;
        if (set + 2 < sets) begin(set + 2, f[0], sv[0], before[0]);
        end(set + 1, f[1], sv[1], before[1]);
      }
      round += sets;
      cluster_arrive();                              // (h_last may be h0: written when all have read it)
      cluster_wait();
    } else {
      for (uint32_t tile = 0; tile < tiles; ++tile) {
        float f[N], sv[N];
        const Map<V> own = evaluate(tile, f, sv);
        __syncthreads();
        ask(tile + kAhead);
        if (tile) {
#pragma unroll
          for (int i = 0; i < V; ++i) h[i] = s_state[turn & 1u][lane][i];
        }
#pragma unroll
        for (uint32_t w = 0; w < kGroups - 1; ++w) {
          if (w == group) break;
          const Map<V> m = s_map[turn & 1u][w][lane];
          fma_v<V>(m.a, h, m.b, h);
        }
        ++turn;
        if (group == kGroups - 1) {
          float behind[V];
          fma_v<V>(own.a, h, own.b, behind);
#pragma unroll
          for (int i = 0; i < V; ++i) s_state[turn & 1u][lane][i] = behind[i];      // (read behind the next barrier)
        }
        apply(tile, f, sv, h);
      }
      __syncthreads();
      if (tiles) {
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = s_state[turn & 1u][lane][i];
      }
    }
    if (a.h_last && in && group == 0 && rank == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) a.h_last[(uint64_t)seq * a.width + c + i] = h[i];
    }
  }
  if constexpr (MODE == kBoxes) {
    if (threadIdx.x == 0 && (taken & kGone)) settle_copies<kDepth>(s_full, asked, a.waits.budget_ns);
  }
  if constexpr (CL > 1) {
    cluster_arrive();
    cluster_wait();
  }
}

// One thread per sequence and V columns.
constexpr uint32_t kShortThreads = 128, kShortAhead = 8, kShortBackAhead = 4, kShortBlock = 16;
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
      if (a.marks && r % kMarkRows == 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) a.marks[(mark0 + r / kMarkRows) * a.width + c + i] = h[i];
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
struct ScanBackMaps {
  CUtensorMap gate, value, dy;
};
// With a cluster a tile's rows are evaluated twice, from shared memory: for the maps that the others wait for, and a set later for the results.
template <int DT, int V, int L, int CL, int MODE>
__global__ void __launch_bounds__(kWarps * 32, 2) scan_back_tiled_kernel(const __grid_constant__ ScanBackArgs a, const __grid_constant__ ScanBackMaps maps) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  using S = TileShape<DT, V, L, 3, CL>;
  constexpr uint32_t kDepth = S::kDepth, kGroups = S::kGroups, kTileRows = S::kTileRows, kColumns = S::kColumns;
  constexpr int R = kRows, N = R * V;                // row k's columns at k V
  extern __shared__ __align__(128) unsigned char smem_raw[];
  unsigned char* smem = smem_raw + ((128u - (smem_u32(smem_raw) & 127u)) & 127u);
  __shared__ __align__(16) Map<V> s_map[2][kGroups][L], s_back[2][kGroups][L];       // of the states, and of the gradient
  __shared__ float s_carry[2][L][V];                // what leaves a tile towards the past, of the first group; in a cluster what reaches the CTA's tile
  Exchange<V, CL, L>& s_x = *reinterpret_cast<Exchange<V, CL, L>*>(smem + S::kDepth * S::kStage);
  __shared__ uint64_t s_full[kDepth];
  __shared__ Chosen s_chosen;
  __shared__ int s_gone;
  volatile int* gone = &s_gone;
  const uint32_t lane = threadIdx.x % L, group = threadIdx.x / L, rank = CL > 1 ? cluster_rank() : 0u;
  if (threadIdx.x == 0) {
    s_gone = 0;
    for (uint32_t s = 0; s < kDepth; ++s) mbar_init(&s_full[s], 1u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (MODE == kBoxes) prefetch_map(&maps.gate), prefetch_map(&maps.value), prefetch_map(&maps.dy);
  }
  if constexpr (CL > 1) exchange_begin(s_x, a.waits.missing_maps);
  else __syncthreads();
  pdl_wait();
  pdl_trigger();
  uint32_t round = 0, asked = 0, taken = 0, turn = 0;
  const uint64_t stride = gridDim.x / CL;
  for (uint64_t item = blockIdx.x / CL; item < a.items; item += stride) {
    uint32_t seq = (uint32_t)(item / a.slabs), first, count;
    const uint32_t col0 = (uint32_t)(item % a.slabs) * kColumns, c = col0 + lane * V;
    if (CL == 1 && a.by_length) {
      longest_first(a.spans, seq, reinterpret_cast<uint32_t*>(s_map), &s_chosen);
      seq = s_chosen.sequence, first = s_chosen.first, count = s_chosen.count;
    } else {
      a.spans.of(seq, &first, &count);
    }
    const bool in = c < a.width;
    T* dgate = static_cast<T*>(a.dgate) + (uint64_t)first * a.ld_dgate + c;
    T* dvalue = static_cast<T*>(a.dvalue) + (uint64_t)first * a.ld_dvalue + c;
    const float* marks = a.marks + first_mark(seq, first) * a.width + c;
    const uint32_t tiles = (count + kTileRows - 1) / kTileRows, sets = (tiles + CL - 1) / CL;
    // sets are counted from the last one: set n holds the tiles (sets - 1 - n) CL + 0 .. CL - 1
    const T* gate = static_cast<const T*>(a.gate) + (uint64_t)first * a.ld_gate + c;
    const T* value = static_cast<const T*>(a.value) + (uint64_t)first * a.ld_value + c;
    const T* dy = static_cast<const T*>(a.dy) + (uint64_t)first * a.ld_dy + c;
    typename P::Raw held[MODE == kRegisters ? 3 : 1][MODE == kRegisters ? R : 1];
    const auto ask = [&](uint32_t n) {               // all threads
      const uint32_t tile = (sets - 1u - n) * CL + rank, s = asked % kDepth;
      const bool there = n < sets && tile < tiles;
      if constexpr (MODE == kBoxes) {
        if (threadIdx.x != 0 || !there || (taken & kGone)) return;
        const int32_t row = (int32_t)(first + tile * kTileRows);
        mbar_arrive_expect_tx(&s_full[s], S::kStage + a.waits.missing_copies);
        tile_load(smem + s * S::kStage, &maps.gate, (int32_t)col0, row, &s_full[s]);
        tile_load(smem + s * S::kStage + S::kInput, &maps.value, (int32_t)col0, row, &s_full[s]);
        tile_load(smem + s * S::kStage + 2 * S::kInput, &maps.dy, (int32_t)col0, row, &s_full[s]);
        ++asked;
      } else {
        const uint32_t r0 = tile * kTileRows + group * R, most = in && there && r0 < count ? count - r0 : 0u;
        const T *from_g = gate + (uint64_t)r0 * a.ld_gate, *from_v = value + (uint64_t)r0 * a.ld_value, *from_d = dy + (uint64_t)r0 * a.ld_dy;
        if constexpr (MODE == kOwnCopies) {
          own_rows<T, V, L>(smem + s * S::kStage, from_g, a.ld_gate, most);
          own_rows<T, V, L>(smem + s * S::kStage + S::kInput, from_v, a.ld_value, most);
          own_rows<T, V, L>(smem + s * S::kStage + 2 * S::kInput, from_d, a.ld_dy, most);
          copies_commit();
        } else {
          held_rows<P>(held[0], from_g, a.ld_gate, most);
          held_rows<P>(held[1], from_v, a.ld_value, most);
          held_rows<P>(held[2], from_d, a.ld_dy, most);
        }
        if (there) ++asked;
      }
    };
    // (registers:) what has been asked for into its stage
    const auto settle = [&](uint32_t s) {
#pragma unroll
      for (uint32_t input = 0; input < 3; ++input) {
        typename P::Raw* to = reinterpret_cast<typename P::Raw*>(smem + s * S::kStage + input * S::kInput) + group * R * L + lane;
#pragma unroll
        for (int k = 0; k < R; ++k) to[k * L] = held[input][k];
      }
    };
    // With a cluster a set's tile is read again one set later: while the maps of set n are made, n and n - 1 hold a stage each and n + 1 may be
    // on its way.
    constexpr uint32_t kAhead = MODE == kRegisters ? 1 : CL > 1 ? kDepth - 2 : kDepth;
    for (uint32_t n = 0; n < kAhead; ++n) ask(n);
    float carry[V];                                  // f[t+1] dh[t+1] of the row behind the tile, or the cluster's tiles
#pragma unroll
    for (int i = 0; i < V; ++i) carry[i] = taken & kGone ? NAN : in && a.dh_last ? a.dh_last[(uint64_t)seq * a.width + c + i] : 0.f;
    struct Rows {
      float f[N], s[N], v[N], d[N];
    };
    const auto rows_of = [&](uint32_t tile) {
      const uint32_t r0 = tile * kTileRows + group * R;
      return tile < tiles && r0 < count ? min((uint32_t)R, count - r0) : 0u;
    };
    const auto read = [&](uint32_t stage, uint32_t rows, Rows& x) __attribute__((always_inline)) {
      if (rows) {
        const T* from = reinterpret_cast<const T*>(smem + stage * S::kStage) + (group * R * L + lane) * V;
        float g[N];
#pragma unroll
        for (int k = 0; k < R; ++k) {
          P::widen(*reinterpret_cast<const typename P::Raw*>(from + k * L * V), g + k * V);
          P::widen(*reinterpret_cast<const typename P::Raw*>(from + S::kInput / sizeof(T) + k * L * V), x.v + k * V);
          P::widen(*reinterpret_cast<const typename P::Raw*>(from + 2 * S::kInput / sizeof(T) + k * L * V), x.d + k * V);
        }
        gates_of<DT>(g, x.f, x.s);
      }
      if (rows < R) {                                // behind the sequence: nothing changes
#pragma unroll
        for (int e = 0; e < N; ++e) {
          if (e / V >= (int)rows) x.f[e] = 1.f, x.s[e] = x.v[e] = x.d[e] = 0.f;
        }
      }
    };
    // Leaves the maps of this group's rows for the others: h -> A h + B of the states, and of the gradient C = sum of d[k] f[0] .. f[k], which is
    // A times what reaches the last row, plus C, at the first.  Returns the latter.
    const auto leave = [&](const Rows& x) __attribute__((always_inline)) {
      Map<V> m, b;
      float sv[N];
      times(x.s, x.v, sv);
#pragma unroll
      for (int i = 0; i < V; ++i) m.a[i] = x.f[i], m.b[i] = sv[i], b.b[i] = 0.f;
      fma_v<V>(m.a, x.d, b.b, b.b);
#pragma unroll
      for (int k = 1; k < R; ++k) {
        fma_v<V>(x.f + k * V, m.b, sv + k * V, m.b);
        mul_v<V>(x.f + k * V, m.a, m.a);
        fma_v<V>(m.a, x.d + k * V, b.b, b.b);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) b.a[i] = m.a[i];
      s_map[turn & 1u][group][lane] = m;
      s_back[turn & 1u][group][lane] = b;
      return b;
    };
    // the state at the last mark before this group's rows
    const uint32_t group0 = group / kMarkGroups * kMarkGroups;
    const auto mark_of = [&](uint32_t tile, float (&h)[V]) {
      const uint32_t r0 = tile * kTileRows + group0 * R;
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = in && tile < tiles && r0 < count ? marks[(uint64_t)(r0 / kMarkRows) * a.width + i] : 0.f;
    };
    const auto wait = [&](uint32_t tile, uint32_t* stage) {
      *stage = taken % kDepth;
      if constexpr (MODE == kOwnCopies) copies_wait<(int)kAhead - 1>();
      if (tile >= tiles) return;
      if constexpr (MODE == kBoxes) {
        if (!wait_for(&s_full[*stage], (taken / kDepth) & 1u, gone, a.waits.budget_ns, taken)) {
          spoil_rows<L>(smem + *stage * S::kStage + S::kInput);
          spoil_rows<L>(smem + *stage * S::kStage + 2 * S::kInput);
        }
      }
      if constexpr (MODE == kRegisters) settle(*stage);
      ++taken;
    };
    // from there to the state before this group's rows
    const auto state_of = [&](float (&h)[V]) __attribute__((always_inline)) {
#pragma unroll
      for (uint32_t n = 0; n < kMarkGroups - 1; ++n) {
        if (group0 + n == group) break;
        const Map<V> m = s_map[turn & 1u][group0 + n][lane];
        fma_v<V>(m.a, h, m.b, h);
      }
    };
    // g: what reaches this group's last row from behind it
    const auto write = [&](uint32_t tile, Rows& x, float (&h)[V], float (&g)[V]) __attribute__((always_inline)) {
      const uint32_t rows = in ? rows_of(tile) : 0u, r0 = tile * kTileRows + group * R;
      float sv[N];
      times(x.s, x.v, sv);
#pragma unroll
      for (int k = 0; k < R; ++k) {
#pragma unroll
        for (int i = 0; i < V; ++i) x.v[k * V + i] = h[i] - x.v[k * V + i];
        fma_v<V>(x.f + k * V, h, sv + k * V, h);
      }
      times(x.v, x.f, x.v);
      T *to_g = dgate + (uint64_t)(r0 + R - 1) * a.ld_dgate, *to_v = dvalue + (uint64_t)(r0 + R - 1) * a.ld_dvalue;
#pragma unroll
      for (int k = R - 1; k >= 0; --k) {
        float dg[V], dv[V], dh[V];
        add_v<V>(x.d + k * V, g, dh);
        mul_v<V>(x.s + k * V, dh, dv);
        mul_v<V>(x.f + k * V, dh, g);
        mul_v<V>(x.v + k * V, dv, dg);
        if (k < (int)rows) {
          P::store(to_g, P::narrow(dg));
          P::store(to_v, P::narrow(dv));
        }
        to_g -= a.ld_dgate, to_v -= a.ld_dvalue;
      }
    };
    if constexpr (CL > 1) {
      float h[V], next_h[V];
      Map<V> behind, next_behind;                    // of the tile's rows behind this group's
      uint32_t stage = 0, next_stage = 0;
      // one warp joins the cluster's maps of a set and leaves what reaches this CTA's tile for all (read behind the next barrier)
      const auto join = [&](uint32_t n) __attribute__((always_inline)) {
        if (threadIdx.x >= 32u) return;
        float g[V];
        exchange_fold<V, CL, true>(s_x, rank, round + n, gone, a.waits.budget_ns, taken, g, carry);
#pragma unroll
        for (int i = 0; i < V; ++i) s_carry[n & 1u][lane][i] = g[i];
      };
      const auto start = [&](uint32_t n) __attribute__((always_inline)) {
        const uint32_t tile = (sets - 1u - n) * CL + rank;
        mark_of(tile, next_h);
        wait(tile, &next_stage);
        Map<V> own;
        {
          Rows x;
          read(next_stage, rows_of(tile), x);
          own = leave(x);
        }
        if (n) join(n - 1);
        __syncthreads();
        // (all are past finish of set n - 2: its stage is free)
        ask(n + kAhead);
        next_behind = identity<V>();
#pragma unroll
        for (uint32_t w = kGroups - 1; w > 0; --w) {
          if (w == group) break;
          append(next_behind, s_back[turn & 1u][w][lane]);
        }
        state_of(next_h);
        ++turn;
        if (group == 0) {
          Map<V> all = next_behind;
          append(all, own);
          exchange_send(s_x, rank, round + n, all);
        }
      };
      for (uint32_t n = 0; n <= sets && sets; ++n) {
        // the maps of set n go out while set n - 1 is finished
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = next_h[i];
        behind = next_behind, stage = next_stage;
        if (n < sets) {
          start(n);
        } else {
          join(n - 1);
          __syncthreads();
        }
        if (n == 0) continue;
        const uint32_t tile = (sets - n) * CL + rank;
        float g[V];
        fma_v<V>(behind.a, s_carry[(n - 1) & 1u][lane], behind.b, g);
        if (rows_of(tile)) {
          Rows x;
          read(stage, rows_of(tile), x);
          write(tile, x, h, g);
        }
      }
      round += sets;
      cluster_arrive();                              // (dh0 may be dh_last: written when all have read it)
      cluster_wait();
    } else {
      for (uint32_t n = 0; n < sets; ++n) {
        const uint32_t tile = sets - 1u - n;
        Rows x;
        float h[V];
        uint32_t stage;
        mark_of(tile, h);
        wait(tile, &stage);
        read(stage, rows_of(tile), x);
        const Map<V> own = leave(x);
        __syncthreads();
        ask(n + kAhead);
        if (n) {
#pragma unroll
          for (int i = 0; i < V; ++i) carry[i] = s_carry[turn & 1u][lane][i];
        }
#pragma unroll
        for (uint32_t w = kGroups - 1; w > 0; --w) {
          if (w == group) break;
          const Map<V> m = s_back[turn & 1u][w][lane];
          fma_v<V>(m.a, carry, m.b, carry);
        }
        state_of(h);
        ++turn;
        if (group == 0) {
          float before[V];
          fma_v<V>(own.a, carry, own.b, before);
#pragma unroll
          for (int i = 0; i < V; ++i) s_carry[turn & 1u][lane][i] = before[i];       // (read behind the next barrier)
        }
        write(tile, x, h, carry);
      }
      __syncthreads();
      if (sets) {
#pragma unroll
        for (int i = 0; i < V; ++i) carry[i] = s_carry[turn & 1u][lane][i];
      }
    }
    if (a.dh0 && in && group == 0 && rank == 0) {
#pragma unroll
      for (int i = 0; i < V; ++i) a.dh0[(uint64_t)seq * a.width + c + i] = carry[i];
    }
  }
  if constexpr (MODE == kBoxes) {
    if (threadIdx.x == 0 && (taken & kGone)) settle_copies<kDepth>(s_full, asked, a.waits.budget_ns);
  }
  if constexpr (CL > 1) {
    cluster_arrive();
    cluster_wait();
  }
}

// One thread per sequence and V columns: kShortBlock rows at a time from the last, first forward from the nearest mark through their states, which are
// kept in shared memory, each thread its own, then back through the gradient.
template <int DT, int V>
__global__ void __launch_bounds__(kShortThreads) scan_back_short_kernel(const __grid_constant__ ScanBackArgs a) {
  using P = Piece<DT, V>;
  using T = typename Elem<DT>::type;
  extern __shared__ __align__(16) unsigned char smem_raw[];
  float* states = reinterpret_cast<float*>(smem_raw) + threadIdx.x * V;      // of row k at k kShortThreads V
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
      const uint32_t r0 = (end - 1) / kShortBlock * kShortBlock, mark = r0 / kMarkRows * kMarkRows;
      float h[V];
#pragma unroll
      for (int i = 0; i < V; ++i) h[i] = marks[(uint64_t)(mark / kMarkRows) * a.width + i];
      for (uint32_t r = mark; r < end; r += kShortBackAhead) {
        typename P::Raw x_raw[kShortBackAhead], v_raw[kShortBackAhead];
#pragma unroll
        for (uint32_t k = 0; k < kShortBackAhead; ++k) {
          if (r + k >= end) continue;
          x_raw[k] = P::load_kept(gate + (uint64_t)(r + k) * a.ld_gate);
          v_raw[k] = P::load_kept(value + (uint64_t)(r + k) * a.ld_value);
        }
#pragma unroll
        for (uint32_t k = 0; k < kShortBackAhead; ++k) {
          if (r + k >= end) continue;
          float x[V], v[V];
          P::widen(x_raw[k], x);
          P::widen(v_raw[k], v);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float f, s;
            gate_of<DT>(x[i], &f, &s);
            if (r >= r0) states[(r + k - r0) * kShortThreads * V + i] = h[i];
            h[i] = fmaf(f, h[i], s * v[i]);
          }
        }
      }
      const uint32_t rows = end - r0;
      for (uint32_t left = rows; left > 0;) {
        const uint32_t n = min(left, kShortBackAhead);
        typename P::Raw x_raw[kShortBackAhead], v_raw[kShortBackAhead], d_raw[kShortBackAhead];
#pragma unroll
        for (uint32_t k = 0; k < kShortBackAhead; ++k) {
          if (k >= n) continue;
          const uint64_t r = r0 + left - 1 - k;
          x_raw[k] = P::load(gate + r * a.ld_gate);
          v_raw[k] = P::load(value + r * a.ld_value);
          d_raw[k] = P::load(dy + r * a.ld_dy);
        }
#pragma unroll
        for (uint32_t k = 0; k < kShortBackAhead; ++k) {
          if (k >= n) continue;
          const uint32_t at = left - 1 - k;
          float x[V], v[V], d[V], dg[V], dv[V];
          P::widen(x_raw[k], x);
          P::widen(v_raw[k], v);
          P::widen(d_raw[k], d);
#pragma unroll
          for (int i = 0; i < V; ++i) {
            float f, s;
            gate_of<DT>(x[i], &f, &s);
            const float dh = d[i] + g[i];
            dv[i] = s * dh;
            g[i] = f * dh;
            dg[i] = dv[i] * (states[at * kShortThreads * V + i] - v[i]) * f;
          }
          P::store(dgate + (uint64_t)(r0 + at) * a.ld_dgate, P::narrow(dg));
          P::store(dvalue + (uint64_t)(r0 + at) * a.ld_dvalue, P::narrow(dv));
        }
        left -= n;
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
// The launch of a kernel over tiles that copies bring, in clusters of `cluster`.
template <typename Args, typename Maps>
cudaError_t launch_tiled(void (*kernel)(Args, Maps), PerDeviceInt& ready, const Args& a, const Maps& maps, uint32_t bytes, uint32_t cluster, cudaStream_t stream) {
  int dev;
  if (!ready.get(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != cudaSuccess) return e;
    ready.set(dev, 1);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)std::min<uint64_t>(a.items, 1u << 24) * cluster);
  cfg.blockDim = dim3(kWarps * 32);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, maps);
}
uint32_t capped(uint64_t ctas) { return (uint32_t)std::min<uint64_t>(ctas, 1u << 24); }
// Sequences that a thread takes by itself: short ones, where there are threads enough (65536 rows of 512 in 2048 sequences: 46 against 95 us, backward
// 123 against 160; 2000 rows in 50 sequences backward 28 against 13), and those of a few rows.
template <typename Args>
bool short_ones(const Args& a, uint32_t columns) {
  const uint32_t mean = a.spans.rows / a.spans.sequences;
  return mean < kStepRows || (mean < kShortRows && (uint64_t)a.spans.sequences * a.width >= 512ull * sm_count() * columns);
}
template <typename Args>
void cut(Args& a, uint32_t columns) {
  a.slabs = (a.width + columns - 1) / columns;
  a.items = (uint64_t)a.spans.sequences * a.slabs;
  a.by_length = a.spans.offsets && a.spans.sequences > 1 && a.spans.sequences <= std::min(kMostOrdered, a.spans.rows / a.spans.sequences) &&
                a.items > 2ull * sm_count() && a.items <= (uint64_t)kOrderedItems * sm_count();
}
// CTAs per sequence and slab: more while two of them would still fit every SM and each has two tiles or more.
uint32_t choose_cluster(uint64_t items, const Spans& s, uint32_t tile_rows) {
  uint32_t cluster = 1;
  while (cluster < kMostCluster && items * cluster * 2 <= 2ull * sm_count() && s.rows / s.sequences >= 4ull * cluster * tile_rows) cluster *= 2;
  return cluster;
}
// Half as many columns and twice the rows to a tile where wide ones in the largest clusters would leave SMs with one CTA or none (one sequence of
// 65536 rows of 1024: 103 us; with wide ones in clusters of 16, which an SM does not take two of, 283).
template <typename Args>
bool narrow_tiles(const Args& a, uint32_t columns) {
  return (uint64_t)a.spans.sequences * ((a.width + columns - 1) / columns) * kMostCluster <= (uint64_t)sm_count() && a.spans.rows / a.spans.sequences >= 8u * kMarkRows;
}
// Rows that tiled copies take: the map's box is the tile.
template <int DT, typename Shape>
bool encode_rows(CUtensorMap* map, const void* p, uint64_t ld, const Spans& s, uint32_t width) {
  constexpr uint64_t item = sizeof(typename Elem<DT>::type);
  return encode_matrix(map, p, (s.rows > 1 ? ld : (width + 7) / 8 * 8) * item, width, s.rows, Shape::kColumns, Shape::kTileRows, DT);
}
bool tiles_take(const void* p, uint64_t ld, uint64_t rows, size_t item) { return aligned_to(p, 16) && (rows <= 1 || ld * item % 16 == 0); }
template <int DT, int V, int L, int CL>
cudaError_t forward_in(const ScanArgs& a, const ScanMaps& m, bool boxes, cudaStream_t stream) {
  static PerDeviceInt ready[2];
  constexpr uint32_t bytes = TileShape<DT, V, L, 2, CL>::kBytes;
  if constexpr (V * sizeof(typename Elem<DT>::type) < 4) {
    return launch_tiled<ScanArgs, ScanMaps>(scan_tiled_kernel<DT, V, L, CL, kRegisters>, ready[0], a, m, bytes, CL, stream);
  } else {
    return launch_tiled<ScanArgs, ScanMaps>(boxes ? scan_tiled_kernel<DT, V, L, CL, kBoxes> : scan_tiled_kernel<DT, V, L, CL, kOwnCopies>, ready[boxes], a, m, bytes, CL, stream);
  }
}
template <int DT, int V, int L>
cudaError_t forward_tiled(ScanArgs a, bool boxes, cudaStream_t stream) {
  using S = TileShape<DT, V, L, 2, 1>;
  cut(a, S::kColumns);
  ScanMaps m;
  std::memset(&m, 0, sizeof(m));
  if (boxes && (!encode_rows<DT, S>(&m.gate, a.gate, a.ld_gate, a.spans, a.width) || !encode_rows<DT, S>(&m.value, a.value, a.ld_value, a.spans, a.width))) return cudaErrorInvalidValue;
  switch (choose_cluster(a.items, a.spans, S::kTileRows)) {
    case 1: return forward_in<DT, V, L, 1>(a, m, boxes, stream);
    case 2: return forward_in<DT, V, L, 2>(a, m, boxes, stream);
    case 4: return forward_in<DT, V, L, 4>(a, m, boxes, stream);
    default: return forward_in<DT, V, L, 8>(a, m, boxes, stream);
  }
}
template <int DT>
cudaError_t launch_forward(ScanArgs a, bool two, cudaStream_t stream) {
  constexpr size_t item = sizeof(typename Elem<DT>::type);
  constexpr int W = item == 2 ? 2 : 1;
  if (short_ones(a, two ? W : 1)) {
    cut(a, two ? W : 1);
    const dim3 grid(capped((a.items + kShortThreads - 1) / kShortThreads)), block(kShortThreads);
    return two ? launch_dependent(scan_short_kernel<DT, W>, grid, block, 0, stream, a) : launch_dependent(scan_short_kernel<DT, 1>, grid, block, 0, stream, a);
  }
  if (two || item == 4) {
    const bool boxes = tiles_take(a.gate, a.ld_gate, a.spans.rows, item) && tiles_take(a.value, a.ld_value, a.spans.rows, item);
    return narrow_tiles(a, 32 * W) ? forward_tiled<DT, W, 16>(a, boxes, stream) : forward_tiled<DT, W, 32>(a, boxes, stream);
  }
  return forward_tiled<DT, 1, 32>(a, false, stream);      // single columns of 16 bits: rows that start anywhere
}
template <int DT, int V, int L, int CL>
cudaError_t backward_in(const ScanBackArgs& a, const ScanBackMaps& m, bool boxes, cudaStream_t stream) {
  static PerDeviceInt ready[2];
  constexpr uint32_t bytes = TileShape<DT, V, L, 3, CL>::kBytes;
  if constexpr (V * sizeof(typename Elem<DT>::type) < 4) {
    return launch_tiled<ScanBackArgs, ScanBackMaps>(scan_back_tiled_kernel<DT, V, L, CL, kRegisters>, ready[0], a, m, bytes, CL, stream);
  } else {
    return launch_tiled<ScanBackArgs, ScanBackMaps>(boxes ? scan_back_tiled_kernel<DT, V, L, CL, kBoxes> : scan_back_tiled_kernel<DT, V, L, CL, kOwnCopies>, ready[boxes], a, m, bytes, CL, stream);
  }
}
template <int DT, int V, int L>
cudaError_t backward_tiled(ScanBackArgs a, bool boxes, cudaStream_t stream) {
  using S = TileShape<DT, V, L, 3, 1>;
  cut(a, S::kColumns);
  ScanBackMaps m;
  std::memset(&m, 0, sizeof(m));
  if (boxes && (!encode_rows<DT, S>(&m.gate, a.gate, a.ld_gate, a.spans, a.width) || !encode_rows<DT, S>(&m.value, a.value, a.ld_value, a.spans, a.width) || !encode_rows<DT, S>(&m.dy, a.dy, a.ld_dy, a.spans, a.width))) return cudaErrorInvalidValue;
  switch (choose_cluster(a.items, a.spans, S::kTileRows)) {
    case 1: return backward_in<DT, V, L, 1>(a, m, boxes, stream);
    case 2: return backward_in<DT, V, L, 2>(a, m, boxes, stream);
    case 4: return backward_in<DT, V, L, 4>(a, m, boxes, stream);
    default: return backward_in<DT, V, L, 8>(a, m, boxes, stream);
  }
}
template <int DT>
cudaError_t launch_backward(ScanBackArgs a, bool two, cudaStream_t stream) {
  constexpr size_t item = sizeof(typename Elem<DT>::type);
  constexpr int W = item == 2 ? 2 : 1;
  if (short_ones(a, two ? W : 1)) {
    cut(a, two ? W : 1);
    const dim3 grid(capped((a.items + kShortThreads - 1) / kShortThreads)), block(kShortThreads);
    constexpr uint32_t bytes = kShortBlock * kShortThreads * 4;     // of one column
    return two ? launch_dependent(scan_back_short_kernel<DT, W>, grid, block, W * bytes, stream, a)
               : launch_dependent(scan_back_short_kernel<DT, 1>, grid, block, bytes, stream, a);
  }
  if (two || item == 4) {
    const bool boxes = tiles_take(a.gate, a.ld_gate, a.spans.rows, item) && tiles_take(a.value, a.ld_value, a.spans.rows, item) && tiles_take(a.dy, a.ld_dy, a.spans.rows, item);
    return narrow_tiles(a, 32 * W) ? backward_tiled<DT, W, 16>(a, boxes, stream) : backward_tiled<DT, W, 32>(a, boxes, stream);
  }
  return backward_tiled<DT, 1, 32>(a, false, stream);      // single columns of 16 bits: rows that start anywhere
}

int check_shape(uint64_t rows, uint64_t sequences, uint64_t width, int dtype, const void* offsets, int offset_bits) {
  if (!is_dtype(dtype) || (offset_bits != 32 && offset_bits != 64)) return GD_ERR_INVALID_ARG;
  if (rows >> 31 || sequences >> 31 || width >> 31) return GD_ERR_TOO_LARGE;
  if (offsets ? !aligned_to(offsets, (size_t)offset_bits / 8) : sequences && rows % sequences) return GD_ERR_INVALID_ARG;
  if (!offsets && !sequences && rows) return GD_ERR_INVALID_ARG;
  return GD_OK;
}

constexpr Waits kWaits{kWaitBudgetNs, 0, 0};
int forward(const gd_recurrence_forward_args* g, const Waits& waits, cudaStream_t stream) {
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
  a.waits = waits;
  a.width = (uint32_t)g->width;
  // two 16-bit columns a thread where rows take 4-byte accesses
  const auto pairs = [&](const void* p, uint64_t ld) { return in_pieces(p, ld, g->rows, g->width, item, 2); };
  const bool two = g->width % 2 == 0 && pairs(g->gate, g->ld_gate) && pairs(g->value, g->ld_value) && pairs(g->y, g->ld_y);
  ProfileScope ps(stream, PT_RECURRENCE);
  cudaError_t e;
  if (g->dtype == GD_DTYPE_FP32) e = launch_forward<GD_DTYPE_FP32>(a, false, stream);
  else e = g->dtype == GD_DTYPE_BF16 ? launch_forward<GD_DTYPE_BF16>(a, two, stream) : launch_forward<GD_DTYPE_FP16>(a, two, stream);
  if (e != cudaSuccess) return GD_ERR_CUDA;
  note_launches(1);
  return GD_OK;
}

int backward(const gd_recurrence_backward_args* g, const Waits& waits, cudaStream_t stream) {
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
  a.waits = waits;
  a.width = (uint32_t)width;
  const auto pairs = [&](const void* p, uint64_t ld) { return in_pieces(p, ld, rows, width, item, 2); };
  const bool two = g->width % 2 == 0 && pairs(g->dy, g->ld_dy) && pairs(g->gate, g->ld_gate) && pairs(g->value, g->ld_value) && pairs(g->dgate, g->ld_dgate) && pairs(g->dvalue, g->ld_dvalue);
  ProfileScope ps(stream, PT_RECURRENCE_BACK);
  cudaError_t e;
  if (g->dtype == GD_DTYPE_FP32) e = launch_backward<GD_DTYPE_FP32>(a, false, stream);
  else e = g->dtype == GD_DTYPE_BF16 ? launch_backward<GD_DTYPE_BF16>(a, two, stream) : launch_backward<GD_DTYPE_FP16>(a, two, stream);
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
  *rows_out = rows / gd::kMarkRows + sequences;
  return GD_OK;
}
int gd_recurrence_forward(const gd_recurrence_forward_args* a, void* stream) { return gd::forward(a, gd::kWaits, (cudaStream_t)stream); }
int gd_recurrence_backward(const gd_recurrence_backward_args* a, void* stream) { return gd::backward(a, gd::kWaits, (cudaStream_t)stream); }

int gd_selftest_recurrence_wait(void* workspace, size_t workspace_bytes, int which, uint64_t budget_ns, void* stream) {
  using namespace gd;
  // 8192 rows: one sequence in a cluster, or, by one CTA, the first of many by their number, of which the others are empty
  constexpr uint64_t rows = 8192, width = 8, many = 64, matrix = rows * width * 2, offsets = 0, marks = 1024, gate = 8192, value = gate + matrix, dy = value + matrix,
                     first = dy + matrix, second = first + matrix, end = second + matrix;
  static_assert(marks + (rows / kMarkRows + many) * width * 4 <= gate && offsets + (many + 1) * 4 <= marks, "the parts of the workspace");
  if (which < 0 || which > 3) return GD_ERR_INVALID_ARG;
  if (!workspace || !aligned_to(workspace, 256) || workspace_bytes < end) return GD_ERR_WORKSPACE;
  unsigned char* base = (unsigned char*)workspace;
  if (cudaMemsetAsync(base, 0, end, (cudaStream_t)stream) != cudaSuccess) return GD_ERR_CUDA;
  if (cudaMemsetAsync(base + offsets + 4, 0x7F, many * 4, (cudaStream_t)stream) != cudaSuccess) return GD_ERR_CUDA;      // (behind the rows: cut to them)
  const bool maps = (which & 1) != 0;
  const Waits waits{budget_ns, maps ? 0u : 8u, maps ? 8u : 0u};
  const auto common = [&](auto& a) {
    a.rows = rows, a.width = width, a.sequences = maps ? 1 : many;
    a.dtype = GD_DTYPE_BF16, a.offset_bits = 32, a.offsets = maps ? nullptr : base + offsets;
    a.gate = base + gate, a.value = base + value;
    a.ld_gate = a.ld_value = width;
    a.marks = (float*)(base + marks);
  };
  if (which < 2) {
    gd_recurrence_forward_args a;
    std::memset(&a, 0, sizeof(a));
    common(a);
    a.y = base + first, a.ld_y = width;
    return gd::forward(&a, waits, (cudaStream_t)stream);
  }
  gd_recurrence_backward_args a;
  std::memset(&a, 0, sizeof(a));
  common(a);
  a.dy = base + dy, a.dgate = base + first, a.dvalue = base + second;
  a.ld_dy = a.ld_dgate = a.ld_dvalue = width;
  return gd::backward(&a, waits, (cudaStream_t)stream);
}

}  // extern "C"
