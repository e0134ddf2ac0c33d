// Embedding lookup with scaling and its gradient by sorted tokens (gd_embedding_forward, gd_embedding_backward).
//
// The lookup is a gather: bound by the bytes, rows read and written in pieces.
//
// The gradient sorts the positions by their id - a stable radix sort of (id, position), digits of up to nine bits - and sums the
// rows of equal ids in ascending order of their positions, so that nothing is added by atomics and every row of the gradient is
// written by one sum.  Most of the gradient is the zeros of ids that do not occur (85000 x 500 in fp32: 170 MB, 26 us, for 4000 positions), and
// the sort is all latency: the launches that sort have CTAs that sort and CTAs that write a share of the zeros meanwhile.
// Measured: that case 37 us (22 without zeros); 131072 positions over 32000 x 1024 113 us, of which the sums take 70 = 5.7 TB/s, the sort 27
// and the join of long runs 15; lookup of 131072 rows of 1024 59 us.
//
// Sums: the sorted list in chunks of kChunk positions, a CTA per chunk and block of columns.  A run of equal ids that ends in the
// chunk after the one it begins in belongs to the latter whole; a longer one leaves the sum of its part of each chunk in the workspace, and the
// next launch joins those, in order.
#include <algorithm>
#include <cstring>

#include "gd_layers.cuh"

namespace gd {
namespace {

constexpr uint32_t kDigitBits = 9, kDigits = 1u << kDigitBits;
constexpr uint32_t kOnePer = 8, kOneThreads = 1024, kOneMost = kOneThreads * kOnePer;           // the sort of one CTA: positions a thread ranks
constexpr uint32_t kTilePer = 4, kTileThreads = 512, kSortTile = kTileThreads * kTilePer;       // the sort of many: each takes a share of whole tiles
constexpr uint32_t kMostTiles = 128;                   // (every one reads the counts of all)
constexpr uint32_t kChunk = 32, kShortChunk = 8;       // positions of a chunk; of lists that one CTA sorts (more CTAs, each with less to wait for)
constexpr uint32_t kFillCtasPerSm = 2;
// Zeros of many bytes under the sort of one CTA: the launch that sorts writes those of the first rows, the one that sums the
// rest, of rows that no id has (85000 x 500 in fp32, 4000 positions: 40 us where the sorting launch wrote them all).
constexpr uint64_t kManyZeros = 32ull << 20, kMostTouched = 1ull << 20;
constexpr double kFirstZeros = 0.6;
// Under the sort of many the zeros cost it their bytes at 8 TB/s.  Where there are positions enough for most rows, the launch that sums writes those of
// the others alone, before all else (131072 positions over 32000 x 1024: 113 us and 124 with all zeros under the sort, ids evenly spread 97 and 116; 40000
// over 85000 x 500 71 and 65).
constexpr uint64_t kDense = 2;         // positions to a row of the table

// ---------------------------------------------------------------- lookup
// A group of `lanes` neighbouring threads (a power of two, up to a warp) takes a row, pieces of up to 16 bytes, kLookAhead of them in hand; the next
// row's id is asked for before this one's pieces.
struct EmbedArgs {
  const void* table;
  const void* ids;
  void* y;
  uint64_t ld_table, ld_y, vocab;
  int64_t ignore_index;
  uint32_t tokens, pieces;     // rows, and pieces of a row
  uint32_t lanes, id_bits;
  float scale;
};
__device__ __forceinline__ int64_t id_at(const void* ids, uint64_t i, uint32_t bits) {
  return bits == 64 ? static_cast<const int64_t*>(ids)[i] : (int64_t)static_cast<const int32_t*>(ids)[i];
}
constexpr uint32_t kLookThreads = 256, kLookAhead = 4;
template <int DT, int OT, int V>
__global__ void __launch_bounds__(kLookThreads) embed_kernel(const __grid_constant__ EmbedArgs a) {
  using P = Piece<DT, V>;
  using Q = Piece<OT, V>;
  pdl_wait();
  pdl_trigger();
  const uint32_t t = blockIdx.x * kLookThreads + threadIdx.x, lane = t & (a.lanes - 1u), step = gridDim.x * kLookThreads / a.lanes;
  uint32_t r = t / a.lanes;
  int64_t next = r < a.tokens ? id_at(a.ids, r, a.id_bits) : 0;
  for (; r < a.tokens; r += step) {
    const int64_t id = next;
    if (r + step < a.tokens) next = id_at(a.ids, r + step, a.id_bits);
    auto* y = static_cast<typename Elem<OT>::type*>(a.y) + r * a.ld_y;
    if (id != a.ignore_index && id >= 0 && (uint64_t)id < a.vocab) {
      const auto* from = static_cast<const typename Elem<DT>::type*>(a.table) + (uint64_t)id * a.ld_table;
      for (uint32_t c = lane; c < a.pieces; c += kLookAhead * a.lanes) {
        typename P::Raw raw[kLookAhead];
#pragma unroll
        for (uint32_t u = 0; u < kLookAhead; ++u)
          if (c + u * a.lanes < a.pieces) raw[u] = P::load_kept(from + (c + u * a.lanes) * V);
#pragma unroll
        for (uint32_t u = 0; u < kLookAhead; ++u) {
          if (c + u * a.lanes >= a.pieces) continue;
          float x[V];
          P::widen(raw[u], x);
#pragma unroll
          for (int i = 0; i < V; ++i) x[i] *= a.scale;
          Q::store(y + (c + u * a.lanes) * V, Q::narrow(x));
        }
      }
    } else {                                      // padding, or an id that is not in the table
      float x[V];
#pragma unroll
      for (int i = 0; i < V; ++i) x[i] = id == a.ignore_index ? 0.f : NAN;
      for (uint32_t c = lane; c < a.pieces; c += a.lanes) Q::store(y + c * V, Q::narrow(x));
    }
  }
}

// ---------------------------------------------------------------- zeros
// The zeros of `rows` rows of `width` elements, `ld` apart: the share of CTA `cta` of `ctas`, in units of 16 bytes where the rows lie one
// behind the other (the few bytes before and after by the first CTA), else a row at a time.
struct Fill {
  void* p;
  uint64_t ld, rows;
  uint32_t width, item;
};
__device__ __forceinline__ void fill_zeros(const Fill& f, uint64_t cta, uint64_t ctas) {
  const uint32_t tid = threadIdx.x, threads = blockDim.x;
  if (f.ld == f.width || f.rows == 1) {
    const uint64_t bytes = f.rows * f.width * f.item, head = min((uint64_t)(16u - ((uint32_t)(uintptr_t)f.p & 15u)) & 15u, bytes);
    unsigned char* base = static_cast<unsigned char*>(f.p);
    const uint64_t vecs = (bytes - head) / 16u, tail = head + vecs * 16u;
    uint4* at = reinterpret_cast<uint4*>(base + head);
    const uint64_t v0 = vecs * cta / ctas, v1 = vecs * (cta + 1) / ctas;
    for (uint64_t v = v0 + tid; v < v1; v += threads) __stcs(at + v, make_uint4(0u, 0u, 0u, 0u));
    if (cta == 0) {
      // (element sizes of 2 and 4: two bytes at a time)
      for (uint64_t b = 2 * tid; b < head; b += 2 * threads) *reinterpret_cast<uint16_t*>(base + b) = 0;
      for (uint64_t b = tail + 2 * tid; b < bytes; b += 2 * threads) *reinterpret_cast<uint16_t*>(base + b) = 0;
    }
    return;
  }
  for (uint64_t r = cta; r < f.rows; r += ctas) {
    if (f.item == 4) {
      float* row = static_cast<float*>(f.p) + r * f.ld;
      for (uint32_t c = tid; c < f.width; c += threads) row[c] = 0.f;
    } else {
      uint16_t* row = static_cast<uint16_t*>(f.p) + r * f.ld;
      for (uint32_t c = tid; c < f.width; c += threads) row[c] = 0;
    }
  }
}
// The zeros of the rows [first, end) that no id has: those whose bit of `touched` is not set, a row to a warp, or, without such bits, that are not among
// the n sorted keys, which a warp looks for 32 at a time.
struct FillRest {
  const uint32_t* touched;
  uint32_t first, end;
};
__device__ __forceinline__ void fill_untouched(const Fill& f, const FillRest& rest, const uint32_t* keys, uint32_t n, uint32_t cta, uint32_t ctas) {
  const uint32_t lane = threadIdx.x & 31u, warps = blockDim.x / 32u, bytes = f.width * f.item, each = rest.touched ? 1u : 32u;
  for (uint64_t r0 = rest.first + (uint64_t)(cta * warps + threadIdx.x / 32u) * each; r0 < rest.end; r0 += (uint64_t)ctas * warps * each) {
    const uint64_t mine = r0 + lane;
    bool none = lane < each && mine < rest.end;
    if (none && rest.touched) {
      none = !(rest.touched[mine >> 5] >> (mine & 31u) & 1u);
    } else if (none) {
      uint32_t from = 0, to = n;                     // the first key that is not below it
      while (from < to) {
        const uint32_t half = from + (to - from) / 2u;
        if (keys[half] < mine) from = half + 1u;
        else to = half;
      }
      none = from == n || keys[from] != mine;
    }
    for (uint32_t left = __ballot_sync(0xFFFFFFFFu, none); left; left &= left - 1u) {
      unsigned char* row = static_cast<unsigned char*>(f.p) + (r0 + __ffs(left) - 1u) * f.ld * f.item;
      if ((((uintptr_t)row | bytes) & 15u) == 0) {
        for (uint32_t b = lane * 16u; b < bytes; b += 512u) __stcs(reinterpret_cast<uint4*>(row + b), make_uint4(0u, 0u, 0u, 0u));
      } else if ((((uintptr_t)row | bytes) & 3u) == 0) {
        for (uint32_t b = lane * 4u; b < bytes; b += 128u) *reinterpret_cast<uint32_t*>(row + b) = 0u;
      } else {
        for (uint32_t b = lane * 2u; b < bytes; b += 64u) *reinterpret_cast<uint16_t*>(row + b) = 0;
      }
    }
  }
}
__global__ void __launch_bounds__(512) fill_kernel(const __grid_constant__ Fill f) {
  pdl_wait();
  pdl_trigger();
  fill_zeros(f, blockIdx.x, gridDim.x);
}

// ---------------------------------------------------------------- sort
struct SortArgs {
  const void* ids;             // the first pass reads these ...
  const uint32_t* keys_in;     // ... the others these
  const uint32_t* at_in;
  uint32_t* keys_out;
  uint32_t* at_out;
  uint32_t* hist;              // [tiles][kDigits]: of this pass
  uint32_t* next_hist;         // of the next one, counted while this one places (NULL: there is none)
  uint32_t* splits;            // splits[0]: how many chunks begin a run that is joined later, zeroed here
  int64_t ignore_index;
  uint32_t n, vocab, id_bits;
  uint32_t shift, bits;        // the pass's digit
  uint32_t passes;             // of the sort of one CTA
  uint32_t tiles, per_tile;    // CTAs that sort, positions each takes (a multiple of kSortTile)
  Fill fill;                   // fill.p NULL: nothing
  uint32_t fill_part, fill_parts;      // which share of the zeros this launch writes
  uint32_t* touched;           // of the sort of one CTA: a bit for every row that is summed into, or NULL
};
// what a position is sorted by: its id, or `vocab`, behind all others
__device__ __forceinline__ uint32_t key_of(const SortArgs& a, uint32_t i) {
  const int64_t id = id_at(a.ids, i, a.id_bits);
  return id != a.ignore_index && id >= 0 && id < (int64_t)a.vocab ? (uint32_t)id : a.vocab;
}
__device__ __forceinline__ void fill_share(const SortArgs& a, uint32_t sorters) {
  const uint64_t ctas = gridDim.x - sorters;
  fill_zeros(a.fill, (uint64_t)a.fill_part * ctas + (blockIdx.x - sorters), ctas * a.fill_parts);
}

// In-place exclusive sums of a[0 .. kDigits) by the first kDigits threads; all threads call it.
__device__ __forceinline__ uint32_t digit_scan(uint32_t x, uint32_t* s_warp) {
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  uint32_t inc = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t y = __shfl_up_sync(0xFFFFFFFFu, inc, o);
    if ((int)lane >= o) inc += y;
  }
  if (lane == 31u) s_warp[warp] = inc;
  __syncthreads();
  uint32_t before = inc - x;
  for (uint32_t w = 0; w < warp; ++w) before += s_warp[w];
  __syncthreads();
  return before;
}

// Stable ranks of THREADS x kPer positions by a digit: rank[u] is the place of position warp * 32 kPer + 32 u + lane among those of the same digit
// in the warps' positions up to it; counts[w][d] afterwards is the number of positions of digit d in the warps before w.
// Returns, in threads d < kDigits, the number of positions of digit d.  `live`: this thread's positions that exist, as bits.
template <uint32_t THREADS, uint32_t kPer>
__device__ __forceinline__ uint32_t rank_digits(const uint32_t (&key)[kPer], uint32_t live, uint32_t shift, uint32_t bits, uint32_t (*counts)[kDigits], uint32_t (&rank)[kPer],
                                                uint32_t rounds = kPer) {
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  for (uint32_t i = threadIdx.x; i < THREADS / 32 * kDigits; i += THREADS) (&counts[0][0])[i] = 0;
  __syncthreads();
#pragma unroll
  for (uint32_t u = 0; u < kPer; ++u) {
    if (u >= rounds) break;
    const bool in = live >> u & 1u;
    const uint32_t d = key[u] >> shift & ((1u << bits) - 1u);
    // the lanes with the same digit, bit by bit (a match over the warp was slower: 25 against 22 us for 4000 positions)
    uint32_t peers = __ballot_sync(0xFFFFFFFFu, in);
#pragma unroll
    for (uint32_t b = 0; b < kDigitBits; ++b) {
      if (b >= bits) break;
      const bool set = d >> b & 1u;
      const uint32_t votes = __ballot_sync(0xFFFFFFFFu, set);
      peers &= set ? votes : ~votes;
    }
    const uint32_t before = in ? counts[warp][d] : 0u;
    __syncwarp();
    rank[u] = before + __popc(peers & lanemask_lt());
    if (in && lane == 31u - __clz(peers)) counts[warp][d] = before + __popc(peers);
    __syncwarp();
  }
  __syncthreads();
  uint32_t total = 0;
  if (threadIdx.x < kDigits) {
#pragma unroll 8
    for (uint32_t w = 0; w < THREADS / 32; ++w) {
      const uint32_t c = counts[w][threadIdx.x];
      counts[w][threadIdx.x] = total;
      total += c;
    }
  }
  return total;
}

// Up to kOneMost positions by one CTA, all passes through shared memory.
struct OneSmem {
  uint32_t counts[kOneThreads / 32][kDigits];
  uint32_t keys[kOneMost], at[kOneMost];
};
__global__ void __launch_bounds__(kOneThreads) sort_one_kernel(const __grid_constant__ SortArgs a) {
  constexpr uint32_t kPer = kOnePer;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ uint32_t s_base[kDigits], s_warp[kOneThreads / 32];
  OneSmem& s = *reinterpret_cast<OneSmem*>(smem);
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x != 0) {
    fill_share(a, 1u);
    return;
  }
  // a warp's positions are neighbours: as many rounds of 32 as there are positions for all warps
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, rounds = (a.n + kOneThreads - 1) / kOneThreads, first = warp * 32u * rounds + lane;
  if (threadIdx.x == 0) a.splits[0] = 0;
  uint32_t key[kPer], at[kPer], rank[kPer], live = 0;
#pragma unroll
  for (uint32_t u = 0; u < kPer; ++u) {
    const uint32_t i = first + 32u * u;
    const bool in = u < rounds && i < a.n;
    live |= (in ? 1u : 0u) << u;
    key[u] = in ? key_of(a, i) : 0u;
    at[u] = i;
  }
  if (a.touched)
    for (uint32_t i = threadIdx.x; i < (a.vocab + 31u) / 32u; i += kOneThreads) a.touched[i] = 0;
  const uint32_t mask = (1u << a.bits) - 1u;
  for (uint32_t p = 0; p < a.passes; ++p) {
    const uint32_t total = rank_digits<kOneThreads, kPer>(key, live, p * a.bits, a.bits, s.counts, rank, rounds);
    const uint32_t base = digit_scan(total, s_warp);
    if (threadIdx.x < kDigits) s_base[threadIdx.x] = base;
    __syncthreads();
#pragma unroll
    for (uint32_t u = 0; u < kPer; ++u) {
      if (!(live >> u & 1u)) continue;
      const uint32_t d = key[u] >> (p * a.bits) & mask, to = s_base[d] + s.counts[warp][d] + rank[u];
      s.keys[to] = key[u], s.at[to] = at[u];
    }
    __syncthreads();
    if (p + 1 == a.passes) break;
#pragma unroll
    for (uint32_t u = 0; u < kPer; ++u) {
      const uint32_t i = first + 32u * u;
      if (live >> u & 1u) key[u] = s.keys[i], at[u] = s.at[i];
    }
  }
  for (uint32_t i = threadIdx.x; i < a.n; i += kOneThreads) {
    const uint32_t k = s.keys[i];
    a.keys_out[i] = k;
    a.at_out[i] = s.at[i];
    if (a.touched && k < a.vocab && (i == 0 || s.keys[i - 1] != k)) atomicOr(&a.touched[k >> 5], 1u << (k & 31u));
  }
}

// More positions: one launch counts the first digits of every share, then one per pass places the positions and counts the next digits of the
// shares they come to (whole numbers: the order of these additions does not matter).
__global__ void __launch_bounds__(kTileThreads) sort_count_kernel(const __grid_constant__ SortArgs a) {
  __shared__ uint32_t s_count[kDigits];
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x >= a.tiles) {
    fill_share(a, a.tiles);
    return;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.splits[0] = 0;
  for (uint32_t d = threadIdx.x; d < kDigits; d += kTileThreads) s_count[d] = 0;
  __syncthreads();
  const uint64_t i0 = (uint64_t)blockIdx.x * a.per_tile, i1 = min(i0 + a.per_tile, (uint64_t)a.n);
  const uint32_t mask = (1u << a.bits) - 1u;
#pragma unroll 4
  for (uint64_t i = i0 + threadIdx.x; i < i1; i += kTileThreads) atomicAdd(&s_count[key_of(a, (uint32_t)i) & mask], 1u);
  __syncthreads();
  for (uint32_t d = threadIdx.x; d < kDigits; d += kTileThreads) {
    a.hist[blockIdx.x * kDigits + d] = s_count[d];
    for (uint32_t p = 1; p < a.passes; ++p) a.hist[(p * kMostTiles + blockIdx.x) * kDigits + d] = 0;
  }
}
struct TileSmem {
  uint32_t counts[kTileThreads / 32][kDigits];
};
template <bool FIRST>
__global__ void __launch_bounds__(kTileThreads, 2) sort_place_kernel(const __grid_constant__ SortArgs a) {
  static_assert(kTileThreads == kDigits, "a thread per digit");
  constexpr uint32_t kPer = kTilePer;
  __shared__ TileSmem s;
  __shared__ uint32_t s_base[kDigits], s_warp[kTileThreads / 32];
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x >= a.tiles) {
    fill_share(a, a.tiles);
    return;
  }
  const uint32_t tid = threadIdx.x, lane = tid & 31u, warp = tid >> 5, mask = (1u << a.bits) - 1u;
  const uint64_t i0 = (uint64_t)blockIdx.x * a.per_tile, i1 = min(i0 + a.per_tile, (uint64_t)a.n);
  uint32_t key[kPer], at[kPer], rank[kPer], live = 0;
  const auto take = [&](uint64_t from) {
    live = 0;
#pragma unroll
    for (uint32_t u = 0; u < kPer; ++u) {
      const uint64_t i = from + warp * 32u * kPer + 32u * u + lane;
      const bool in = i < i1;
      live |= (in ? 1u : 0u) << u;
      key[u] = !in ? 0u : FIRST ? key_of(a, (uint32_t)i) : a.keys_in[i];
      at[u] = !in ? 0u : FIRST ? (uint32_t)i : a.at_in[i];
    }
  };
  take(i0);
  uint32_t before = 0, total = 0;      // positions of digit `tid` in the shares before this one, and in all
  constexpr uint32_t kBatch = 32;      // loads in hand: the loop is all latency
  for (uint32_t t0 = 0; t0 < a.tiles; t0 += kBatch) {
    uint32_t c[kBatch];
#pragma unroll
    for (uint32_t t = 0; t < kBatch; ++t) c[t] = t0 + t < a.tiles ? __ldcg(&a.hist[(t0 + t) * kDigits + tid]) : 0u;
#pragma unroll
    for (uint32_t t = 0; t < kBatch; ++t) {
      before += t0 + t < blockIdx.x ? c[t] : 0u;
      total += c[t];
    }
  }
  s_base[tid] = digit_scan(total, s_warp) + before;
  for (uint64_t from = i0; from < i1; from += kSortTile) {
    if (from != i0) take(from);
    const uint32_t here = rank_digits<kTileThreads, kPer>(key, live, a.shift, a.bits, s.counts, rank);
    __syncthreads();
#pragma unroll
    for (uint32_t u = 0; u < kPer; ++u) {
      if (!(live >> u & 1u)) continue;
      const uint32_t d = key[u] >> a.shift & mask, to = s_base[d] + s.counts[warp][d] + rank[u];
      a.keys_out[to] = key[u];
      a.at_out[to] = at[u];
      if (a.next_hist) atomicAdd(&a.next_hist[to / a.per_tile * kDigits + (key[u] >> (a.shift + a.bits) & mask)], 1u);
    }
    __syncthreads();
    s_base[tid] += here;
  }
}

// ---------------------------------------------------------------- sums
struct SumArgs {
  const void* dy;
  const uint32_t* keys;
  const uint32_t* at;
  void* dtable;
  float* part;                 // [chunks][2][part_ld]: of the run that came in, of the run that goes on
  uint32_t* splits;            // [0]: how many, [1 ..]: chunks that begin a run that is joined later
  uint64_t ld_dy, ld_dtable;
  uint32_t n, vocab, width, part_ld;
  float scale;
  uint32_t accumulate;
  Fill fill;                   // zeros that are left to the launch that sums: its first `fillers` CTAs (in x) write those of `rest`
  FillRest rest;
  uint32_t fillers;
};
template <int GT, int V>
__device__ __forceinline__ void put_row(const SumArgs& a, uint32_t key, uint32_t c, float (&sum)[V]) {
  using Q = Piece<GT, V>;
  auto* to = static_cast<typename Elem<GT>::type*>(a.dtable) + (uint64_t)key * a.ld_dtable + c;
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] *= a.scale;
  if (a.accumulate) {
    float old[V];
    Q::widen(*reinterpret_cast<const typename Q::Raw*>(to), old);
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] += old[i];
  }
  *reinterpret_cast<typename Q::Raw*>(to) = Q::narrow(sum);
}
constexpr uint32_t kSumAhead = 8;
template <int DT, int GT, int V, uint32_t kChunk>
__global__ void __launch_bounds__(256) sum_kernel(const __grid_constant__ SumArgs a) {
  using P = Piece<DT, V>;
  __shared__ uint32_t s_key[3 * kChunk + 2], s_at[2 * kChunk];      // s_key[j]: of sorted position i0 - kChunk - 1 + j
  pdl_wait();
  pdl_trigger();
  if (blockIdx.x < a.fillers) {
    fill_untouched(a.fill, a.rest, a.keys, a.n, blockIdx.y * a.fillers + blockIdx.x, a.fillers * gridDim.y);
    return;
  }
  const uint32_t chunk = blockIdx.x - a.fillers, i0 = chunk * kChunk, i1 = min(i0 + kChunk, a.n), tid = threadIdx.x;
  constexpr uint32_t kNone = 0xFFFFFFFFu;                            // (a key is at most vocab < 2^31)
  for (uint32_t j = tid; j < 3 * kChunk + 2; j += blockDim.x) {
    const int64_t i = (int64_t)i0 - kChunk - 1 + j;
    s_key[j] = i >= 0 && i < (int64_t)a.n ? a.keys[i] : kNone;
  }
  for (uint32_t j = tid; j < 2 * kChunk; j += blockDim.x) s_at[j] = (uint64_t)i0 + j < a.n ? a.at[i0 + j] : 0u;
  __syncthreads();
  const uint32_t* key = s_key + kChunk + 1;                          // key[j]: of position i0 + j, j from -kChunk - 1 to 2 kChunk
  const uint32_t c = (blockIdx.y * blockDim.x + tid) * V, here = i1 - i0;
  // What of this chunk's neighbours' is its own: a run that came in is its to sum only where it is one of those that are joined later; a run that
  // goes on is summed to its end if that lies in the next chunk.
  uint32_t j = 0, end = here;
  bool came = false, goes = false;                                   // the first sum is a part, the last one is
  if (key[-1] == key[0] && key[0] != kNone) {
    came = key[-(int)kChunk - 1] == key[0] || (here == kChunk && key[kChunk] == key[0]);
    if (!came)
      while (j < here && key[j] == key[-1]) ++j;
  }
  const uint32_t last = key[here - 1];
  if (here == kChunk && key[kChunk] == last && key[-1] != last) {
    goes = key[2 * kChunk] == last;
    if (!goes)
      while (key[end] == last) ++end;                                // (ends before 2 kChunk: key[2 kChunk] is another)
    if (goes && last < a.vocab && tid == 0 && blockIdx.y == 0) a.splits[1u + atomicAdd(&a.splits[0], 1u)] = chunk;
  }
  while (end > j && key[end - 1] >= a.vocab) --end;                  // positions without a row of the table
  if (c >= a.width || j >= end) return;
  const auto* dy = static_cast<const typename Elem<DT>::type*>(a.dy) + c;
  float* part = a.part + (uint64_t)chunk * 2 * a.part_ld + c;
  float sum[V];
#pragma unroll
  for (int i = 0; i < V; ++i) sum[i] = 0.f;
  while (j < end) {
    typename P::Raw raw[kSumAhead];
#pragma unroll
    for (uint32_t u = 0; u < kSumAhead; ++u)
      if (j + u < end) raw[u] = P::load(dy + (uint64_t)s_at[j + u] * a.ld_dy);
#pragma unroll
    for (uint32_t u = 0; u < kSumAhead; ++u) {
      if (j + u >= end) continue;
      float x[V];
      P::widen(raw[u], x);
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] += x[i];
      const uint32_t k = key[j + u];
      if (j + u + 1 < end && key[j + u + 1] == k) continue;
      // the run's last row here
      if ((came && k == key[-1]) || (goes && k == last)) {
        Piece<GD_DTYPE_FP32, V>::store(part + (came && k == key[-1] ? 0u : a.part_ld), Piece<GD_DTYPE_FP32, V>::narrow(sum));
      } else {
        put_row<GT, V>(a, k, c, sum);
      }
#pragma unroll
      for (int i = 0; i < V; ++i) sum[i] = 0.f;
    }
    j += kSumAhead;
  }
}

// The runs of more than two chunks: the part of the chunk they begin in, then those of the chunks that follow, shared out to the warps in order.
// (500000 positions over 32000 x 128: 115 us, of 8 warps 128; of 32 131072 over 32000 x 1024 takes 126 in place of 113)
constexpr uint32_t kJoinWarps = 16;
template <int GT, int V>
__global__ void __launch_bounds__(32 * kJoinWarps) sum_join_kernel(const __grid_constant__ SumArgs a, uint32_t chunk_rows) {
  using F = Piece<GD_DTYPE_FP32, V>;                  // (the parts' rows are multiples of four apart)
  __shared__ float s_sum[kJoinWarps][32 * V];
  __shared__ uint32_t s_more;
  pdl_wait();
  pdl_trigger();
  const uint32_t count = a.splits[0], lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, c = (blockIdx.y * 32u + lane) * V;
  for (uint32_t e = blockIdx.x; e < count; e += gridDim.x) {
    const uint32_t chunk = a.splits[1u + e], key = a.keys[(uint64_t)chunk * chunk_rows + chunk_rows - 1];
    // how many chunks follow that begin inside the run
    uint32_t more = 0;
    for (bool on = true; on; ) {
      if (threadIdx.x == 0) s_more = 0;
      __syncthreads();
      const uint64_t i = ((uint64_t)chunk + 1 + more + threadIdx.x) * chunk_rows;
      const uint32_t inside = __ballot_sync(0xFFFFFFFFu, i < a.n && a.keys[i < a.n ? i : 0] == key);
      if (lane == 0) atomicAdd(&s_more, (uint32_t)__popc(inside));
      __syncthreads();
      const uint32_t got = s_more;
      more += got;
      on = got == 32 * kJoinWarps;
      __syncthreads();
    }
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.f;
    if (c < a.width) {
      if (warp == 0) {
        F::widen(F::load_kept(a.part + ((uint64_t)chunk * 2 + 1) * a.part_ld + c), sum);
      }
      const uint32_t m0 = (uint64_t)more * warp / kJoinWarps, m1 = (uint64_t)more * (warp + 1) / kJoinWarps;
      constexpr uint32_t kInHand = 8;
      for (uint32_t m = m0; m < m1; m += kInHand) {
        typename F::Raw raw[kInHand];
#pragma unroll
        for (uint32_t u = 0; u < kInHand; ++u)
          raw[u] = m + u < m1 ? F::load_kept(a.part + ((uint64_t)chunk + 1 + m + u) * 2 * a.part_ld + c) : F::none();
#pragma unroll
        for (uint32_t u = 0; u < kInHand; ++u) {
          float x[V];
          F::widen(raw[u], x);
#pragma unroll
          for (int i = 0; i < V; ++i) sum[i] += x[i];
        }
      }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) s_sum[warp][lane * V + i] = sum[i];
    __syncthreads();
    if (warp == 0 && c < a.width) {
#pragma unroll
      for (uint32_t w = 1; w < kJoinWarps; ++w) {
#pragma unroll
        for (int i = 0; i < V; ++i) sum[i] += s_sum[w][lane * V + i];
      }
      put_row<GT, V>(a, key, c, sum);
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------- host side
uint64_t up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }
uint32_t bits_of(uint64_t x) {      // of the largest key
  uint32_t b = 1;
  while (x >> b) ++b;
  return b;
}
uint32_t chunk_of(uint64_t n) { return n <= kOneMost ? kShortChunk : kChunk; }
// Where everything is in the workspace.
struct Layout {
  uint64_t keys[2], at[2], hist, splits, touched, part, part_ld, end;
  Layout(uint64_t n, uint64_t vocab, uint64_t width) {
    uint64_t o = 0;
    const auto take = [&](uint64_t bytes) {
      const uint64_t p = o;
      o += up(bytes, 256);
      return p;
    };
    const bool one = n <= kOneMost;
    for (int i = 0; i < 2; ++i) keys[i] = i && one ? 0 : take(4 * n), at[i] = i && one ? 0 : take(4 * n);
    hist = take(one ? 0 : 4ull * kMostTiles * kDigits * 4);        // (31 bits are four passes)
    const uint32_t chunk = chunk_of(n);
    const uint64_t chunks = (n + chunk - 1) / chunk;
    splits = take(4 * (chunks + 1));
    touched = take(one && vocab <= kMostTouched ? (vocab + 31) / 32 * 4 : 0);
    part_ld = up(width, 4);
    part = take(n > 2 * chunk ? chunks * 2 * part_ld * 4 : 0);
    end = std::max<uint64_t>(o, 256);
  }
};
// Of any number of positions up to n: short lists are cut into shorter chunks, so the longest of them may want more than n do.
uint64_t workspace_up_to(uint64_t n, uint64_t vocab, uint64_t width) {
  return std::max(Layout(n, vocab, width).end, Layout(std::min<uint64_t>(n, kOneMost), vocab, width).end);
}

template <int DT, int OT, int V>
cudaError_t launch_pieces(EmbedArgs a, uint32_t width, cudaStream_t stream) {
  a.pieces = width / V;
  a.lanes = 1;
  while (a.lanes < 32 && a.lanes < a.pieces) a.lanes *= 2;
  const uint64_t ctas = ((uint64_t)a.tokens * a.lanes + kLookThreads - 1) / kLookThreads;
  return launch_dependent(embed_kernel<DT, OT, V>, dim3((uint32_t)std::min<uint64_t>(ctas, (uint64_t)sm_count() * 8)), dim3(kLookThreads), 0, stream, a);
}
template <int DT, int OT>
cudaError_t launch_lookup(const EmbedArgs& a, const gd_embedding_forward_args* g, cudaStream_t stream) {
  constexpr size_t in = sizeof(typename Elem<DT>::type), out = sizeof(typename Elem<OT>::type);
  const uint32_t width = (uint32_t)g->width;
  const auto takes = [&](uint32_t v) { return in_pieces(a.table, a.ld_table, 2, width, in, v) && in_pieces(a.y, a.ld_y, g->tokens, width, out, v); };
  if constexpr (in == 2 && out == 2) {
    if (takes(8)) return launch_pieces<DT, OT, 8>(a, width, stream);
  }
  return takes(4) ? launch_pieces<DT, OT, 4>(a, width, stream) : takes(2) ? launch_pieces<DT, OT, 2>(a, width, stream) : launch_pieces<DT, OT, 1>(a, width, stream);
}

int forward(const gd_embedding_forward_args* g, cudaStream_t stream) {
  if (!g || !is_dtype(g->table_dtype) || !is_dtype(g->y_dtype) || (g->id_bits != 32 && g->id_bits != 64)) return GD_ERR_INVALID_ARG;
  if (g->y_dtype != g->table_dtype && g->y_dtype != GD_DTYPE_FP32 && g->table_dtype != GD_DTYPE_FP32) return GD_ERR_INVALID_ARG;
  if (g->tokens >> 31 || g->vocab >> 31 || g->width >> 20) return GD_ERR_TOO_LARGE;
  if (g->tokens == 0 || g->width == 0) return GD_OK;
  if (!g->ids || !aligned_to(g->ids, (size_t)g->id_bits / 8) || !good_matrix(g->y, g->ld_y, g->tokens, g->width, dtype_bytes(g->y_dtype)) ||
      (g->vocab && !good_matrix(g->table, g->ld_table, g->vocab, g->width, dtype_bytes(g->table_dtype))))
    return GD_ERR_INVALID_ARG;
  EmbedArgs a;
  std::memset(&a, 0, sizeof(a));
  a.table = g->table, a.ld_table = g->vocab > 1 ? g->ld_table : g->width;
  a.ids = g->ids, a.id_bits = (uint32_t)g->id_bits;
  a.y = g->y, a.ld_y = g->ld_y;
  a.vocab = g->vocab, a.tokens = (uint32_t)g->tokens;
  a.ignore_index = g->ignore_index;
  a.scale = g->scale;
  ProfileScope ps(stream, PT_EMBED);
  cudaError_t e;
  constexpr int F = GD_DTYPE_FP32, B = GD_DTYPE_BF16, H = GD_DTYPE_FP16;
  if (g->table_dtype == F)
    e = g->y_dtype == F ? launch_lookup<F, F>(a, g, stream) : g->y_dtype == B ? launch_lookup<F, B>(a, g, stream) : launch_lookup<F, H>(a, g, stream);
  else if (g->table_dtype == B)
    e = g->y_dtype == F ? launch_lookup<B, F>(a, g, stream) : launch_lookup<B, B>(a, g, stream);
  else
    e = g->y_dtype == F ? launch_lookup<H, F>(a, g, stream) : launch_lookup<H, H>(a, g, stream);
  if (e != cudaSuccess) return GD_ERR_CUDA;
  note_launches(1);
  return GD_OK;
}

cudaError_t launch_sort(SortArgs& a, const Layout& l, unsigned char* ws, const uint32_t** keys, const uint32_t** at, cudaStream_t stream) {
  const uint32_t bits = bits_of(a.vocab);
  a.passes = (bits + kDigitBits - 1) / kDigitBits;
  a.bits = (bits + a.passes - 1) / a.passes;
  const auto keys_at = [&](uint32_t i) { return reinterpret_cast<uint32_t*>(ws + l.keys[i]); };
  const auto at_at = [&](uint32_t i) { return reinterpret_cast<uint32_t*>(ws + l.at[i]); };
  const uint64_t fill_bytes = a.fill.p ? a.fill.rows * a.fill.width * a.fill.item : 0;
  // CTAs that write zeros, no more than have 4 KB each
  const auto fillers = [&](uint32_t launches, uint32_t per_sm) { return (uint32_t)std::min<uint64_t>((fill_bytes + launches * 4096ull - 1) / (launches * 4096ull), (uint64_t)sm_count() * per_sm); };
  if (a.n <= kOneMost) {
    static PerDeviceInt ready;
    int dev;
    if (!ready.get(&dev)) {
      const cudaError_t e = cudaFuncSetAttribute(sort_one_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(OneSmem));
      if (e != cudaSuccess) return e;
      ready.set(dev, 1);
    }
    a.keys_out = keys_at(0), a.at_out = at_at(0);
    a.fill_part = 0, a.fill_parts = 1;
    *keys = a.keys_out, *at = a.at_out;
    ProfileScope ps(stream, PT_EMBED_SORT);
    note_launches(1);
    return launch_dependent(sort_one_kernel, dim3(1 + std::min(fillers(1, 1), (uint32_t)std::max(1, sm_count() - 1))), dim3(kOneThreads), sizeof(OneSmem), stream, a);
  }
  const uint32_t whole = (a.n + kSortTile - 1) / kSortTile, per = (whole + kMostTiles - 1) / kMostTiles;
  a.per_tile = per * kSortTile;
  a.tiles = (whole + per - 1) / per;
  uint32_t* hist = reinterpret_cast<uint32_t*>(ws + l.hist);
  a.hist = hist;
  a.fill_parts = 1 + a.passes;
  const dim3 grid(a.tiles + fillers(a.fill_parts, kFillCtasPerSm)), block(kTileThreads);
  const auto launch = [&](void (*kernel)(SortArgs)) {
    ProfileScope ps(stream, PT_EMBED_SORT);
    const cudaError_t e = launch_dependent(kernel, grid, block, 0, stream, a);
    if (e == cudaSuccess) note_launches(1);
    return e;
  };
  cudaError_t e = launch(sort_count_kernel);
  if (e != cudaSuccess) return e;
  for (uint32_t p = 0; p < a.passes; ++p) {
    a.shift = p * a.bits;
    a.hist = hist + (uint64_t)p * kMostTiles * kDigits;
    a.next_hist = p + 1 < a.passes ? hist + (uint64_t)(p + 1) * kMostTiles * kDigits : nullptr;
    if (p) a.keys_in = keys_at((p - 1) & 1u), a.at_in = at_at((p - 1) & 1u);
    a.keys_out = keys_at(p & 1u), a.at_out = at_at(p & 1u);
    a.fill_part = p + 1;
    e = launch(p ? sort_place_kernel<false> : sort_place_kernel<true>);
    if (e != cudaSuccess) return e;
  }
  *keys = a.keys_out, *at = a.at_out;
  return cudaSuccess;
}

template <int DT, int GT, int V>
cudaError_t launch_sums(SumArgs a, cudaStream_t stream) {
  const uint32_t pieces = (a.width + V - 1) / V, chunk = chunk_of(a.n), chunks = (a.n + chunk - 1) / chunk;
  const uint32_t threads = std::min(256u, (pieces + 31) / 32 * 32), across = (pieces + threads - 1) / threads;
  const uint32_t left = a.rest.end - a.rest.first;   // rows whose zeros are left to this launch
  const uint32_t fillers = left ? std::min((left + 31) / 32, 1024u * (uint32_t)sm_count() / threads / across + 1) : 0u;
  a.fillers = fillers;
  {
    ProfileScope ps(stream, PT_EMBED_SUM);
    const cudaError_t e = launch_dependent(chunk == kShortChunk ? sum_kernel<DT, GT, V, kShortChunk> : sum_kernel<DT, GT, V, kChunk>, dim3(chunks + fillers, across),
                                           dim3(threads), 0, stream, a);
    if (e != cudaSuccess) return e;
    note_launches(1);
  }
  if (a.n <= 2 * chunk) return cudaSuccess;          // (no run can be longer)
  const uint32_t blocks = (a.width + 32 * V - 1) / (32 * V);
  ProfileScope ps(stream, PT_EMBED_JOIN);
  const cudaError_t e = launch_dependent(sum_join_kernel<GT, V>, dim3(std::min(chunks, std::max(1u, 8u * (uint32_t)sm_count() / blocks)), blocks), dim3(32 * kJoinWarps),
                                         0, stream, a, chunk);
  if (e == cudaSuccess) note_launches(1);
  return e;
}
template <int DT, int GT>
cudaError_t launch_sums_v(const SumArgs& a, cudaStream_t stream) {
  const bool four = in_pieces(a.dy, a.ld_dy, a.n, a.width, sizeof(typename Elem<DT>::type), 4) &&
                    in_pieces(a.dtable, a.ld_dtable, a.vocab, a.width, sizeof(typename Elem<GT>::type), 4);
  return four ? launch_sums<DT, GT, 4>(a, stream) : launch_sums<DT, GT, 1>(a, stream);
}

int backward(const gd_embedding_backward_args* g, cudaStream_t stream) {
  if (!g || g->reserved != 0 || !is_dtype(g->dtype) || (g->dtable_dtype != g->dtype && g->dtable_dtype != GD_DTYPE_FP32) || (g->id_bits != 32 && g->id_bits != 64) ||
      (g->flags & ~(uint32_t)GD_EMBEDDING_ACCUMULATE))
    return GD_ERR_INVALID_ARG;
  const bool accumulate = (g->flags & GD_EMBEDDING_ACCUMULATE) != 0;
  if (accumulate && g->dtable_dtype != GD_DTYPE_FP32) return GD_ERR_INVALID_ARG;
  if (g->tokens >> 31 || g->vocab >> 31 || g->width >> 20) return GD_ERR_TOO_LARGE;
  if (g->vocab == 0 || g->width == 0 || (accumulate && g->tokens == 0)) return GD_OK;
  const size_t item = dtype_bytes(g->dtable_dtype);
  if (!good_matrix(g->dtable, g->ld_dtable, g->vocab, g->width, item)) return GD_ERR_INVALID_ARG;
  Fill fill;
  std::memset(&fill, 0, sizeof(fill));
  fill.p = accumulate ? nullptr : g->dtable, fill.ld = g->ld_dtable, fill.rows = g->vocab, fill.width = (uint32_t)g->width, fill.item = (uint32_t)item;
  if (g->tokens == 0) {
    ProfileScope ps(stream, PT_EMBED_FILL);
    if (launch_dependent(fill_kernel, dim3(4 * sm_count()), dim3(512), 0, stream, fill) != cudaSuccess) return GD_ERR_CUDA;
    note_launches(1);
    return GD_OK;
  }
  if (!g->ids || !aligned_to(g->ids, (size_t)g->id_bits / 8) || !good_matrix(g->dy, g->ld_dy, g->tokens, g->width, dtype_bytes(g->dtype))) return GD_ERR_INVALID_ARG;
  const Layout l(g->tokens, g->vocab, g->width);
  if (!g->workspace || !aligned_to(g->workspace, 256) || g->workspace_bytes < l.end) return GD_ERR_WORKSPACE;
  unsigned char* ws = static_cast<unsigned char*>(g->workspace);
  SortArgs s;
  std::memset(&s, 0, sizeof(s));
  s.ids = g->ids, s.id_bits = (uint32_t)g->id_bits;
  s.ignore_index = g->ignore_index;
  s.n = (uint32_t)g->tokens, s.vocab = (uint32_t)g->vocab;
  s.splits = reinterpret_cast<uint32_t*>(ws + l.splits);
  s.fill = fill;
  SumArgs a;
  std::memset(&a, 0, sizeof(a));
  if (fill.p && s.n <= kOneMost && g->vocab <= kMostTouched && g->vocab * g->width * item >= kManyZeros) {
    s.touched = reinterpret_cast<uint32_t*>(ws + l.touched);
    s.fill.rows = (uint64_t)(kFirstZeros * (double)g->vocab);
    a.fill = fill;
    a.rest = FillRest{s.touched, (uint32_t)s.fill.rows, (uint32_t)g->vocab};
  }
  if (fill.p && s.n > kOneMost && s.n >= kDense * g->vocab) {
    s.fill.p = nullptr;
    a.fill = fill;
    a.rest = FillRest{nullptr, 0u, (uint32_t)g->vocab};
  }
  if (launch_sort(s, l, ws, &a.keys, &a.at, stream) != cudaSuccess) return GD_ERR_CUDA;
  a.dy = g->dy, a.ld_dy = g->ld_dy;
  a.dtable = g->dtable, a.ld_dtable = g->vocab > 1 ? g->ld_dtable : up(g->width, 4);
  a.part = reinterpret_cast<float*>(ws + l.part), a.part_ld = (uint32_t)l.part_ld;
  a.splits = s.splits;
  a.n = s.n, a.vocab = s.vocab, a.width = (uint32_t)g->width;
  a.scale = g->scale;
  a.accumulate = accumulate;
  constexpr int F = GD_DTYPE_FP32, B = GD_DTYPE_BF16, H = GD_DTYPE_FP16;
  cudaError_t e;
  if (g->dtype == F) e = launch_sums_v<F, F>(a, stream);
  else if (g->dtype == B) e = g->dtable_dtype == F ? launch_sums_v<B, F>(a, stream) : launch_sums_v<B, B>(a, stream);
  else e = g->dtable_dtype == F ? launch_sums_v<H, F>(a, stream) : launch_sums_v<H, H>(a, stream);
  return e == cudaSuccess ? GD_OK : GD_ERR_CUDA;
}

}  // namespace
}  // namespace gd

extern "C" {

int gd_embedding_workspace_bytes(uint64_t tokens, uint64_t vocab, uint64_t width, size_t* bytes_out) {
  if (!bytes_out) return GD_ERR_INVALID_ARG;
  if (tokens >> 31 || vocab >> 31 || width >> 20) return GD_ERR_TOO_LARGE;
  *bytes_out = (size_t)gd::workspace_up_to(tokens, vocab, width);
  return GD_OK;
}
int gd_embedding_forward(const gd_embedding_forward_args* a, void* stream) { return gd::forward(a, (cudaStream_t)stream); }
int gd_embedding_backward(const gd_embedding_backward_args* a, void* stream) { return gd::backward(a, (cudaStream_t)stream); }

}  // extern "C"
