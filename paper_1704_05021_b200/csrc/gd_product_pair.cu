// The product for outputs of many tiles: pairs of CTAs on 256 x 256 tiles, one persistent pair per two SMs.
//
// Bound by the tensor cores, if they are fed, and by the power the GPU may draw.  A 128 x 256 x 64 block takes an SM 512 cycles; the
// pair's instruction (cta_group::2) lets each SM bring only its own half of A and of B, 32 KB, so an SM draws 64 bytes per cycle
// from L2 where a tile of its own of that size would draw 96, and 128 x 128 tiles 128.  Ten warps: one thread asks for the copies
// (kStages blocks deep), one thread of the leading CTA issues the products for both, eight warps take finished sums out of tensor
// memory, 128 columns of 32 lanes each, and finish the tile while the next one is summed into the other half of it: 2 x 256
// columns, all there are.  A lane holds a row, so results leave through shared memory: a piece of 32 rows x 128 bytes per warp, two of
// them in turn, stored by the copy engine, which cuts what lies outside the matrix and takes any row pitch that is a multiple of 16 bytes; the
// residual comes in the same way, into the piece the result is then written over.  Stores are cut to whole 16 bytes only (measured: 4096 x 4097
// results in 16 bits put zeros into the seven elements behind each row; loads are cut to the element), so their map ends at the row's last whole 16
// bytes and each lane writes what is left of its row.  Other pitches: element by element, a row at a time.
//
// Tiles are taken in groups of kGroup tile rows, column by column, so that what the pairs read at one time stays in L2.
#include <algorithm>
#include <cstring>

#include "gd_mma.cuh"

namespace gd {
namespace {

constexpr uint32_t kPairWarps = 8;                            // that finish tiles
constexpr uint32_t kPairThreads = (kPairWarps + 2) * 32;
constexpr uint32_t kHalfA = 128 * kBlockK * 2;                // one CTA's half of a block of A
constexpr uint32_t kPieceBytes = 32 * 128;                  // rows x bytes of a piece
template <int BN>
struct PairShape {
  static constexpr uint32_t kHalfB = BN / 2 * kBlockK * 2;
  static constexpr uint32_t kStage = kHalfA + kHalfB;
  static constexpr uint32_t kStages = BN == 256 ? 5 : 6;
  static constexpr uint32_t kBytes = kStages * kStage + kPairWarps * 2 * kPieceBytes + 1024;
};
constexpr uint32_t kGroup = 8;

struct PairArgs {
  CUtensorMap a, b;
  CUtensorMap out, pre, add;      // pieces of the results and of the residual (TILED)
  Epilogue ep;
  int* status;
  uint32_t blocks_k, chain, desc;
  uint32_t tiles_r, tiles_c;
  uint32_t beside;
};

__device__ __forceinline__ void tile_load_pair(void* dst, const CUtensorMap* map, int32_t x, int32_t y, uint32_t barrier) {
  asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
               "l"(map), "r"(x), "r"(y), "r"(barrier)
               : "memory");
}
// b, in both CTAs of the pair, receives one arrive when the products issued so far have been done
__device__ __forceinline__ void mma_commit_pair(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(b)), "h"((uint16_t)3) : "memory");
}
__device__ __forceinline__ void mbar_arrive_peer(uint32_t address) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(address) : "memory");
}

__device__ __forceinline__ void tile_store(const CUtensorMap* map, const void* src, int32_t x, int32_t y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(smem_u32(src)) : "memory");
}
// Closes a group of stores.  Every piece closes one, whether it was stored or lies outside the matrix (an empty group is done at once): the pieces
// take the buffers in turn and stores_read() counts groups, so the two counts have to run together.
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// columns that make up whole 16 bytes of a row
__host__ __device__ constexpr uint32_t whole_columns(uint32_t cols, uint32_t item) { return cols & ~(16u / item - 1u); }
template <int LEFT>
__device__ __forceinline__ void stores_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(LEFT) : "memory"); }   // all but LEFT have left shared memory
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// first row and column tile of the t-th tile: groups of kGroup tile rows, within a group column by column
__device__ __forceinline__ void tile_place(uint32_t t, uint32_t tiles_r, uint32_t tiles_c, uint32_t* r, uint32_t* c) {
  const uint32_t in_group = kGroup * tiles_c, group = t / in_group, rest = t % in_group;
  const uint32_t rows = min(kGroup, tiles_r - group * kGroup);
  *r = group * kGroup + rest % rows;
  *c = rest / rows;
}

// CHAINED: a tile's sum is made of several (fp32 results), joined in registers; otherwise it goes from tensor memory straight out.
// TILED: results and residual go through the copy engine.  WIDE: the results are fp32.
template <int BN, bool A_MN, bool B_MN, bool CHAINED, bool TILED, bool WIDE>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1) product_pair_kernel(const __grid_constant__ PairArgs g) {
  constexpr uint32_t kPairStages = PairShape<BN>::kStages, kPairStage = PairShape<BN>::kStage, kHalf = BN / 2;     // kHalf: columns a warp finishes
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t full[kPairStages], empty[kPairStages], sum_full[2], sum_empty[2], add_full[kPairWarps][2];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  const uint32_t rank = cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const uint32_t tiles = g.tiles_r * g.tiles_c;
  if (tid == 0) {
    for (uint32_t s = 0; s < kPairStages; ++s) mbar_init(&full[s], 1u), mbar_init(&empty[s], 1u);
    for (uint32_t s = 0; s < 2; ++s) mbar_init(&sum_full[s], 1u), mbar_init(&sum_empty[s], 2 * kPairWarps);   // (the leader's: both CTAs' warps)
    for (uint32_t w = 0; w < kPairWarps; ++w) mbar_init(&add_full[w][0], 1u), mbar_init(&add_full[w][1], 1u);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (g.blocks_k) prefetch_map(&g.a), prefetch_map(&g.b);
  }
  if (warp == kPairWarps) tmem_alloc<2>(&s_tmem, 2 * BN);
  fence_before();
  cluster_arrive();                                  // both CTAs' barriers exist before either signals the other's
  cluster_wait();
  fence_after();
  const uint32_t tmem = s_tmem;
  const volatile int* abort = &s_abort;
  bool good = true;
  if (!g.beside) pdl_wait();                         // (the other product's CTAs are past theirs: all have triggered)
  pdl_trigger();

  if (warp == kPairWarps) {                          // copies: each CTA its halves, all counted on the leader's barrier
    if (elect_one()) {
      uint32_t n = 0;
      for (uint32_t t = pair; good && t < tiles; t += pairs) {
        uint32_t tr, tc;
        tile_place(t, g.tiles_r, g.tiles_c, &tr, &tc);
        const int32_t i0 = (int32_t)(tr * 256u + rank * 128u), j0 = (int32_t)(tc * BN + rank * kHalf);
        for (uint32_t k = 0; k < g.blocks_k; ++k, ++n) {
          const uint32_t s = n % kPairStages;
          if (n >= kPairStages && !mbar_wait(&empty[s], (n / kPairStages + 1u) & 1u, abort)) { good = false; break; }
          unsigned char* at = smem + s * kPairStage;
          const uint32_t bar = peer_address(smem_u32(&full[s]), 0);
          const int32_t kc = (int32_t)(k * kBlockK);
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * kPairStage);
          if constexpr (A_MN) {
            tile_load_pair(at, &g.a, i0, kc, bar);
            tile_load_pair(at + 8192, &g.a, i0 + 64, kc, bar);
          } else {
            tile_load_pair(at, &g.a, kc, i0, bar);
          }
          if constexpr (B_MN) {
            tile_load_pair(at + kHalfA, &g.b, j0, kc, bar);
            if constexpr (BN == 256) tile_load_pair(at + kHalfA + 8192, &g.b, j0 + 64, kc, bar);
          } else {
            tile_load_pair(at + kHalfA, &g.b, kc, j0, bar);
          }
        }
      }
      // every block has been used (in the ordinary case): what the CTA asked for has landed, and nothing will still arrive at its barriers
      const int none = 0;
      if (!good) s_abort = 1;
      for (uint32_t u = n > kPairStages ? n - kPairStages : 0u; u < n; ++u) {
        if (good) good = mbar_wait(&empty[u % kPairStages], (u / kPairStages) & 1u, abort);
        else if (rank == 0) (void)mbar_wait(&full[u % kPairStages], (u / kPairStages) & 1u, &none);
      }
    }
  } else if (warp == kPairWarps + 1) {               // products, issued by the leader for both
    if (rank == 0 && elect_one()) {
      uint32_t n = 0, chain = 0;
      for (uint32_t t = pair; good && t < tiles; t += pairs) {
        for (uint32_t k = 0; good && k < g.blocks_k; ++chain) {
          const uint32_t end = min(k + g.chain, g.blocks_k), buf = chain & 1u, sum = tmem + buf * BN;
          if (chain >= 2 && !mbar_wait(&sum_empty[buf], (chain / 2 + 1u) & 1u, abort)) { good = false; break; }
          fence_after();
          for (const uint32_t first = k; k < end; ++k, ++n) {
            const uint32_t s = n % kPairStages;
            if (!mbar_wait(&full[s], (n / kPairStages) & 1u, abort)) { good = false; break; }
            fence_after();
            const uint32_t at = smem_u32(smem + s * kPairStage);
#pragma unroll
            for (uint32_t q = 0; q < kBlockK / 16; ++q) {
              const uint64_t a = operand_desc(at + q * (A_MN ? 2048u : 32u), 8192u);
              const uint64_t b = operand_desc(at + kHalfA + q * (B_MN ? 2048u : 32u), 8192u);
              mma<2>(sum, a, b, g.desc, (k - first) | q);
            }
            mma_commit_pair(&empty[s]);
          }
          if (good) mma_commit_pair(&sum_full[buf]);
        }
      }
      if (!good) s_abort = 1;
    }
  } else {
    // warps w and w + 4 take the lanes of quarter w, half of the columns each
    constexpr uint32_t W = WIDE ? 32 : 64, kPieces = kHalf / W;     // columns of a piece
    const uint32_t quarter = warp & 3u, half = (warp >> 2) * kHalf;
    unsigned char* pieces = smem + kPairStages * kPairStage + warp * 2 * kPieceBytes;
    const Epilogue& ep = g.ep;
    uint32_t chain = 0, add_phase = 0, turn = 0;     // turn: pieces so far; they take the two buffers in turn, across tiles too
    for (uint32_t t = pair; good && t < tiles; t += pairs) {
      uint32_t tr, tc;
      tile_place(t, g.tiles_r, g.tiles_c, &tr, &tc);
      const uint32_t r0 = tr * 256u + rank * 128u + quarter * 32u, c0 = tc * BN + half;
      const uint32_t from = tmem + (quarter * 32u << 16) + half;
      const auto release = [&](uint32_t buf) {       // this warp has read its part of the sum
        fence_before();
        __syncwarp();
        if (elect_one()) mbar_arrive_peer(peer_address(smem_u32(&sum_empty[buf]), 0));
      };
      // Lane l holds the bias of columns 4 l .. 4 l + 3; asked for before the sum is there.
      float bias[4] = {0.f, 0.f, 0.f, 0.f};
      if (TILED && ep.bias) {
#pragma unroll
        for (uint32_t i = 0; i < 4; ++i)
          if (4 * lane < kHalf && c0 + 4 * lane + i < ep.cols) bias[i] = load_as(ep.bias, c0 + 4 * lane + i, ep.bias_dtype);
      }
      const bool through = ep.add && (!WIDE || ep.add_dtype == GD_DTYPE_FP32);      // the residual comes as pieces; one of 16 bits next to fp32 results does not fit
      // The residual of piece p, `ahead` turns from now, into the buffer whose place the result takes (buffer 0 alone where z also needs one).
      const auto ask_add = [&](uint32_t p, uint32_t ahead) {
        const uint32_t at = !WIDE && ep.pre ? 0u : (turn + ahead) & 1u;
        mbar_arrive_expect_tx(&add_full[warp][at], kPieceBytes);
        tile_load(pieces + at * kPieceBytes, &g.add, (int32_t)(c0 + p * W), (int32_t)r0, &add_full[warp][at]);
      };
      // v: the lane's row of piece p
      const auto finish = [&](uint32_t p, float* v) {
        const uint32_t c = c0 + p * W;
        if constexpr (TILED) {
          const uint32_t whole = whole_columns(ep.cols, WIDE ? 4 : 2);
          const bool inside = r0 < ep.rows && c < whole;
          // the row's last columns, short of 16 bytes, from the lane's own row of a piece
          const auto finish_row = [&](void* to, uint64_t ld, const unsigned char* from) {
            if (whole == ep.cols || c >= ep.cols || whole >= c + W || r0 + lane >= ep.rows) return;
            const uint4 q = *reinterpret_cast<const uint4*>(from + ((whole - c) / (W / 8) ^ (lane & 7u)) * 16u);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
            const uint64_t at = (uint64_t)(r0 + lane) * ld + whole;
#pragma unroll
            for (uint32_t i = 0; i < W / 8; ++i) {
              if (whole + i >= ep.cols) continue;
              if constexpr (WIDE) static_cast<uint32_t*>(to)[at + i] = w[i];
              else static_cast<uint16_t*>(to)[at + i] = (uint16_t)(w[i / 2] >> (i & 1u) * 16u);
            }
          };
          const bool two = !WIDE && ep.pre;          // z takes the second buffer
          const uint32_t at = two ? 0u : turn & 1u;
          unsigned char* mine = pieces + at * kPieceBytes + lane * 128u;
          unsigned char* z = pieces + kPieceBytes + lane * 128u;
          if (!through || two) {                     // (with a residual the buffer was free before its copy was asked for)
            if (elect_one()) { if (two) stores_read<0>(); else stores_read<1>(); }
            __syncwarp();
          }
          if (ep.bias) {
#pragma unroll
            for (uint32_t j = 0; j < W; ++j) v[j] += __shfl_sync(0xFFFFFFFFu, bias[j & 3u], (p * W + j) >> 2);
          }
          if constexpr (!WIDE) {
            if (ep.pre) {
#pragma unroll
              for (uint32_t j = 0; j < 8; ++j) *reinterpret_cast<uint4*>(z + (j ^ (lane & 7u)) * 16u) = narrow8(v + 8 * j, ep.dtype);
              finish_row(ep.pre, ep.ld_pre, z);
              fence_async();
              __syncwarp();
              if (elect_one()) {
                if (inside) tile_store(&g.pre, pieces + kPieceBytes, (int32_t)c, (int32_t)r0);
                stores_commit();
              }
            }
          }
          if constexpr (WIDE) {
            if (ep.pre && r0 + lane < ep.rows) {     // 32 columns of 16 bits a lane: two sectors, written directly
              uint16_t* to = static_cast<uint16_t*>(ep.pre) + (uint64_t)(r0 + lane) * ep.ld_pre + c;
#pragma unroll
              for (uint32_t j = 0; j < 4; ++j) {
                if (c + 8 * j + 8 <= ep.cols) {
                  *reinterpret_cast<uint4*>(to + 8 * j) = narrow8(v + 8 * j, ep.dtype);
                } else {
#pragma unroll
                  for (uint32_t i = 0; i < 8; ++i)
                    if (c + 8 * j + i < ep.cols) store_as(to, 8 * j + i, ep.dtype, v[8 * j + i]);
                }
              }
            }
          }
          activate_all<W>(v, ep.activation);
          if constexpr (WIDE) {
            if (ep.add && !through && r0 + lane < ep.rows) {
              const uint16_t* of = static_cast<const uint16_t*>(ep.add) + (uint64_t)(r0 + lane) * ep.ld_add + c;
#pragma unroll
              for (uint32_t j = 0; j < 4; ++j) {
                float w[8] = {};
                if (c + 8 * j + 8 <= ep.cols) {
                  load8_as(of, 8 * j, ep.add_dtype, w);
                } else {
#pragma unroll
                  for (uint32_t i = 0; i < 8; ++i)
                    if (c + 8 * j + i < ep.cols) w[i] = load_as(of, 8 * j + i, ep.add_dtype);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * j + i] += w[i];
              }
            }
          }
          if (through) {
            good = mbar_wait(&add_full[warp][at], add_phase >> at & 1u, abort) && good;
            add_phase ^= 1u << at;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
              const uint4 q = *reinterpret_cast<const uint4*>(mine + (j ^ (lane & 7u)) * 16u);
              if constexpr (WIDE) {
                v[4 * j] += __uint_as_float(q.x), v[4 * j + 1] += __uint_as_float(q.y);
                v[4 * j + 2] += __uint_as_float(q.z), v[4 * j + 3] += __uint_as_float(q.w);
              } else {
                float w[8];
                widen8(q, ep.dtype, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * j + i] += w[i];
              }
            }
          }
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j) {
            uint4* chunk = reinterpret_cast<uint4*>(mine + (j ^ (lane & 7u)) * 16u);
            if constexpr (WIDE)
              *chunk = make_uint4(__float_as_uint(v[4 * j]), __float_as_uint(v[4 * j + 1]), __float_as_uint(v[4 * j + 2]), __float_as_uint(v[4 * j + 3]));
            else
              *chunk = narrow8(v + 8 * j, ep.dtype);
          }
          finish_row(ep.out, ep.ld_out, mine);
          fence_async();
          __syncwarp();
          if (elect_one()) {
            if (inside) tile_store(&g.out, pieces + at * kPieceBytes, (int32_t)c, (int32_t)r0);
            stores_commit();
            if (through && p + 1 < kPieces) {
              if (two) stores_read<0>(); else stores_read<1>();
              ask_add(p + 1, 1);
            }
          }
          ++turn;
        } else {
          // any pitch: a row of the piece at a time, one column per lane, or two neighbours where the rows allow it (512 x 50258 results of
          // depth 512: 54 us one, 37 two; 4000 x 1500 of 1000 24.0 and 22.3, with residual and z 48.5 and 27.7)
          float* piece = reinterpret_cast<float*>(pieces);
          __syncwarp();
#pragma unroll
          for (uint32_t j = 0; j < W / 4; ++j)
            *reinterpret_cast<float4*>(piece + lane * W + (j ^ (lane & 7u)) * 4u) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
          __syncwarp();
          if (!WIDE && ep.pairs) {
            const uint32_t two = c + 2 * lane;
            const float b0 = ep.bias && two < ep.cols ? load_as(ep.bias, two, ep.bias_dtype) : 0.f;
            const float b1 = ep.bias && two + 1 < ep.cols ? load_as(ep.bias, two + 1, ep.bias_dtype) : 0.f;
#pragma unroll 1
            for (uint32_t r = 0; r < 32; r += 8) {   // (eight rows' values first: a store may not be passed by the loads behind it)
              float o[8], q[8];
#pragma unroll
              for (uint32_t u = 0; u < 8; ++u) {
                const float2 f = *reinterpret_cast<const float2*>(piece + (r + u) * W + ((lane >> 1) ^ u) * 4u + (lane & 1u) * 2u);
                o[u] = f.x + b0, q[u] = f.y + b1;
              }
              if (two < ep.cols) finish_columns(ep, r0 + r, two, o, q);
            }
          } else {
#pragma unroll
            for (uint32_t h = 0; h < W; h += 32) {
              const uint32_t one = c + h + lane;
              const bool in = one < ep.cols;
              const float bias = in && ep.bias ? load_as(ep.bias, one, ep.bias_dtype) : 0.f;
#pragma unroll 1
              for (uint32_t r = 0; r < 32; r += 8) {
                float o[8];
#pragma unroll
                for (uint32_t u = 0; u < 8; ++u) o[u] = piece[h + (r + u) * W + ((lane >> 2) ^ u) * 4u + (lane & 3u)] + bias;
                if (in) finish_column(ep, r0 + r, one, o);
              }
            }
          }
        }
      };
      if constexpr (TILED) {
        if (through && elect_one()) {                  // the first piece's residual is under way while the sum is still being made
          stores_read<0>();
          ask_add(0, 0);
        }
      }
      if constexpr (CHAINED) {
        float v[kHalf];
#pragma unroll
        for (uint32_t c = 0; c < kHalf; ++c) v[c] = 0.f;
        for (uint32_t k = 0; k < g.blocks_k; k += g.chain, ++chain) {
          const uint32_t buf = chain & 1u;
          if (!mbar_wait(&sum_full[buf], (chain / 2) & 1u, abort)) { good = false; break; }
          fence_after();
#pragma unroll
          for (uint32_t c = 0; c < kHalf; c += 16) {
            float w[16];
            tmem_load8(from + buf * BN + c, w);
            tmem_load8(from + buf * BN + c + 8, w + 8);
            tmem_ready();
#pragma unroll
            for (int j = 0; j < 16; ++j) v[c + j] += w[j];
          }
          release(buf);
        }
        if (good) {
#pragma unroll
          for (uint32_t p = 0; p < kPieces; ++p) finish(p, v + p * W);
        }
      } else {
        const uint32_t buf = chain & 1u;
        good = mbar_wait(&sum_full[buf], (chain / 2) & 1u, abort);
        ++chain;
        if (good) {
          fence_after();
#pragma unroll 1
          for (uint32_t p = 0; p < kPieces; ++p) {
            float v[W];
#pragma unroll
            for (uint32_t c = 0; c < W; c += 32) tmem_load32(from + buf * BN + p * W + c, v + c);
            tmem_ready();
            if (p + 1 == kPieces) release(buf);
            finish(p, v);
          }
        }
      }
    }
    if constexpr (TILED) {
      if (elect_one()) {
        // (a residual asked for by a tile whose sum never came still has to land)
        const int none = 0;
        if (!good && ep.add && (!WIDE || ep.add_dtype == GD_DTYPE_FP32)) (void)mbar_wait(&add_full[warp][!WIDE && ep.pre ? 0 : turn & 1u], add_phase >> (!WIDE && ep.pre ? 0 : turn & 1u) & 1u, &none, 1000000ull);
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
      }
    }
    if (!good) s_abort = 1;
  }
  if (!good) atomicExch(g.status, GD_ERR_DEVICE_TIMEOUT);
  __syncwarp();
  fence_before();
  cluster_arrive();                                  // neither CTA leaves while the other's products read its memory or its warps signal
  cluster_wait();
  if (warp == kPairWarps) tmem_free<2>(tmem, 2 * BN);
  if (g.beside) pdl_wait();
}

template <int BN, bool A_MN, bool B_MN, bool CHAINED, bool TILED, bool WIDE>
cudaError_t launch_pair(const PairArgs& g, cudaStream_t stream) {
  auto kernel = product_pair_kernel<BN, A_MN, B_MN, CHAINED, TILED, WIDE>;
  static PerDeviceInt ready;
  int dev;
  if (!ready.get(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairShape<BN>::kBytes);
    if (e != cudaSuccess) return e;
    ready.set(dev, 1);
  }
  const uint32_t pairs = std::min<uint64_t>((uint64_t)g.tiles_r * g.tiles_c, (uint64_t)sm_count() / 2);
  return launch_dependent(kernel, dim3(2 * pairs), dim3(kPairThreads), PairShape<BN>::kBytes, stream, g);
}
template <int BN, bool A_MN, bool B_MN>
cudaError_t launch_majors(const PairArgs& g, bool tiled, cudaStream_t stream) {
  const bool chained = g.chain < g.blocks_k;            // (fp32 results only)
  if (g.ep.out_dtype == GD_DTYPE_FP32) {
    if (tiled) return chained ? launch_pair<BN, A_MN, B_MN, true, true, true>(g, stream) : launch_pair<BN, A_MN, B_MN, false, true, true>(g, stream);
    return chained ? launch_pair<BN, A_MN, B_MN, true, false, true>(g, stream) : launch_pair<BN, A_MN, B_MN, false, false, true>(g, stream);
  }
  return tiled ? launch_pair<BN, A_MN, B_MN, false, true, false>(g, stream) : launch_pair<BN, A_MN, B_MN, false, false, false>(g, stream);
}
template <int BN>
cudaError_t launch_bn(const Product& p, const PairArgs& g, bool tiled, cudaStream_t stream) {
  if (p.a.mn_major) return p.b.mn_major ? launch_majors<BN, true, true>(g, tiled, stream) : cudaErrorInvalidValue;   // (no call has A alone transposed)
  return p.b.mn_major ? launch_majors<BN, false, true>(g, tiled, stream) : launch_majors<BN, false, false>(g, tiled, stream);
}

}  // namespace

cudaError_t launch_product_pair(const Product& p, uint32_t bn, cudaStream_t stream) {
  PairArgs g;
  std::memset(&g, 0, sizeof(g));
  if (!encode_operand(&g.a, p.a, p.ep.rows, p.depth, p.a.mn_major ? 64 : 128, p.bf16) ||
      !encode_operand(&g.b, p.b, p.ep.cols, p.depth, p.b.mn_major ? 64 : bn / 2, p.bf16))
    return cudaErrorInvalidValue;
  g.ep = p.ep;
  g.status = p.status;
  g.beside = p.beside;
  g.blocks_k = (p.depth + kBlockK - 1) / kBlockK;
  g.chain = chain_blocks(p);
  g.desc = mma_desc(256, bn, p.bf16, p.a.mn_major, p.b.mn_major);
  g.tiles_r = (p.ep.rows + 255) / 256;
  g.tiles_c = (p.ep.cols + bn - 1) / bn;
  // results and residual as pieces of 32 rows x 128 bytes, where every row starts at a multiple of 16 bytes
  const bool wide = g.ep.out_dtype == GD_DTYPE_FP32, tiled = g.ep.vectors && whole_columns(g.ep.cols, wide ? 4 : 2);
  const uint32_t whole = whole_columns(g.ep.cols, wide ? 4 : 2);
  if (tiled && (!encode_piece(&g.out, g.ep.out, g.ep.ld_out, g.ep, whole, g.ep.out_dtype) ||
                (g.ep.pre && !wide && !encode_piece(&g.pre, g.ep.pre, g.ep.ld_pre, g.ep, whole, g.ep.dtype)) ||
                (g.ep.add && g.ep.add_dtype == g.ep.out_dtype && !encode_piece(&g.add, g.ep.add, g.ep.ld_add, g.ep, g.ep.cols, g.ep.add_dtype))))
    return cudaErrorInvalidValue;
  return bn == 256 ? launch_bn<256>(p, g, tiled, stream) : launch_bn<128>(p, g, tiled, stream);
}

}  // namespace gd
