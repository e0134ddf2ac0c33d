// The product for outputs of many tiles: pairs of CTAs on 256 x 256 tiles, one persistent pair per two SMs.
//
// Bound by the tensor cores, if they are fed.  A 128 x 256 x 64 block takes an SM 512 cycles; the pair's instruction
// (cta_group::2) lets each SM bring only its own half of A and of B, 32 KB, so an SM draws 64 bytes per cycle from L2 where a tile of
// its own of that size would draw 96, and 128 x 128 tiles 128.  Ten warps: one thread asks for the copies (kStages blocks deep),
// one thread of the leading CTA issues the products for both, eight warps take finished sums out of tensor memory into registers, 128
// columns of 32 lanes each, hand the tensor memory back at once and finish the tile while the next one is summed into the other
// half of it: 2 x 256 columns, all there are.  On its way out a piece of 32 x 32 passes through shared memory so that a warp's
// accesses to bias, residual and results run along rows, 64 bytes of 8 rows each.
//
// Tiles are taken in groups of kGroup tile rows, column by column, so that what the pairs read at one time stays in L2.
#include <algorithm>
#include <cstring>

#include "gd_mma.cuh"

namespace gd {
namespace {

constexpr uint32_t kPairWarps = 8;                            // that finish tiles
constexpr uint32_t kPairThreads = (kPairWarps + 2) * 32;
constexpr uint32_t kPairStages = 6;
constexpr uint32_t kHalfBlock = 128 * kBlockK * 2;            // one CTA's half of a block of A or of B
constexpr uint32_t kPairStage = 2 * kHalfBlock;
constexpr uint32_t kPieceBytes = 32 * 32 * 4;
constexpr uint32_t kPairBytes = kPairStages * kPairStage + kPairWarps * kPieceBytes + 1024;
constexpr uint32_t kGroup = 8;

struct PairArgs {
  CUtensorMap a, b;
  Epilogue ep;
  int* status;
  uint32_t blocks_k, chain, desc;
  uint32_t tiles_r, tiles_c;
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

// first row and column tile of the t-th tile: groups of kGroup tile rows, within a group column by column
__device__ __forceinline__ void tile_place(uint32_t t, uint32_t tiles_r, uint32_t tiles_c, uint32_t* r, uint32_t* c) {
  const uint32_t in_group = kGroup * tiles_c, group = t / in_group, rest = t % in_group;
  const uint32_t rows = min(kGroup, tiles_r - group * kGroup);
  *r = group * kGroup + rest % rows;
  *c = rest / rows;
}

// CHAINED: a tile's sum is made of several (fp32 results), joined in registers; otherwise it goes from tensor memory straight out.
template <bool A_MN, bool B_MN, bool CHAINED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1) product_pair_kernel(const __grid_constant__ PairArgs g) {
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t full[kPairStages], empty[kPairStages], sum_full[2], sum_empty[2];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  const uint32_t rank = cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const uint32_t tiles = g.tiles_r * g.tiles_c;
  if (tid == 0) {
    for (uint32_t s = 0; s < kPairStages; ++s) mbar_init(&full[s], 1u), mbar_init(&empty[s], 1u);
    for (uint32_t s = 0; s < 2; ++s) mbar_init(&sum_full[s], 1u), mbar_init(&sum_empty[s], 2 * kPairWarps);   // (the leader's: both CTAs' warps)
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (g.blocks_k) prefetch_map(&g.a), prefetch_map(&g.b);
  }
  if (warp == kPairWarps) tmem_alloc<2>(&s_tmem, 512);
  fence_before();
  cluster_arrive();                                  // both CTAs' barriers exist before either signals the other's
  cluster_wait();
  fence_after();
  const uint32_t tmem = s_tmem;
  const volatile int* abort = &s_abort;
  bool good = true;
  pdl_wait();
  pdl_trigger();

  if (warp == kPairWarps) {                          // copies: each CTA its halves, all counted on the leader's barrier
    if (lane == 0) {
      uint32_t n = 0;
      for (uint32_t t = pair; good && t < tiles; t += pairs) {
        uint32_t tr, tc;
        tile_place(t, g.tiles_r, g.tiles_c, &tr, &tc);
        const int32_t i0 = (int32_t)(tr * 256u + rank * 128u), j0 = (int32_t)(tc * 256u + rank * 128u);
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
            tile_load_pair(at + kHalfBlock, &g.b, j0, kc, bar);
            tile_load_pair(at + kHalfBlock + 8192, &g.b, j0 + 64, kc, bar);
          } else {
            tile_load_pair(at + kHalfBlock, &g.b, kc, j0, bar);
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
    if (lane == 0 && rank == 0) {
      uint32_t n = 0, chain = 0;
      for (uint32_t t = pair; good && t < tiles; t += pairs) {
        for (uint32_t k = 0; good && k < g.blocks_k; ++chain) {
          const uint32_t end = min(k + g.chain, g.blocks_k), buf = chain & 1u, sum = tmem + buf * 256u;
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
              const uint64_t b = operand_desc(at + kHalfBlock + q * (B_MN ? 2048u : 32u), 8192u);
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
    // warps w and w + 4 take the lanes of quarter w, 128 of the 256 columns each
    const uint32_t quarter = warp & 3u, half = (warp >> 2) * 128u;
    float* piece = reinterpret_cast<float*>(smem + kPairStages * kPairStage) + warp * (kPieceBytes / 4);
    uint32_t chain = 0;
    for (uint32_t t = pair; good && t < tiles; t += pairs) {
      uint32_t tr, tc;
      tile_place(t, g.tiles_r, g.tiles_c, &tr, &tc);
      const uint32_t r0 = tr * 256u + rank * 128u + quarter * 32u, c0 = tc * 256u + half;
      // A piece of 32 x 32: each lane puts its row into shared memory, then the warp works along the rows.  A row's 16-byte chunks are
      // XORed with the row's number, so that neither the lanes' rows nor the rows' neighbours meet in a bank.
      const auto put = [&](const float* w) {
        __syncwarp();
#pragma unroll
        for (uint32_t c = 0; c < 8; ++c)
          *reinterpret_cast<float4*>(piece + lane * 32u + (c ^ (lane & 7u)) * 4u) = make_float4(w[4 * c], w[4 * c + 1], w[4 * c + 2], w[4 * c + 3]);
        __syncwarp();
      };
      const auto get8 = [&](uint32_t r, float (&o)[8]) {   // the lane's eight columns of row r
        const uint32_t c = (lane & 3u) * 2u;
        const float4 x = *reinterpret_cast<const float4*>(piece + r * 32u + (c ^ (r & 7u)) * 4u), y = *reinterpret_cast<const float4*>(piece + r * 32u + ((c + 1u) ^ (r & 7u)) * 4u);
        o[0] = x.x, o[1] = x.y, o[2] = x.z, o[3] = x.w, o[4] = y.x, o[5] = y.y, o[6] = y.z, o[7] = y.w;
      };
      // what the epilogue reads is asked for before the sum is there: a lane's eight columns of the bias, its rows of the residual
      const bool fast = g.ep.vectors && r0 + 32 <= g.ep.rows && c0 + 128 <= g.ep.cols, add16 = g.ep.add && g.ep.add_dtype != GD_DTYPE_FP32;
      const uint32_t lr = lane >> 2, lc = (lane & 3u) * 8u;
      float bias[8];
      uint4 add[4];
      const auto fetch = [&](uint32_t q) {
        if (!fast) return;
        if (g.ep.bias) load8_as(g.ep.bias, c0 + 32 * q + lc, g.ep.bias_dtype, bias);
        if (add16) {
#pragma unroll
          for (uint32_t u = 0; u < 4; ++u)
            add[u] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(g.ep.add) + (uint64_t)(r0 + u * 8 + lr) * g.ep.ld_add + c0 + 32 * q + lc);
        }
      };
      const auto finish = [&](uint32_t q) {
        const uint32_t c = c0 + 32 * q + lc;
        if (!fast) {
#pragma unroll 1
          for (uint32_t u = 0; u < 4; ++u) {
            float o[8];
            get8(u * 8 + lr, o);
            finish8(g.ep, r0 + u * 8 + lr, c, o);
          }
          return;
        }
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
          const uint64_t r = r0 + u * 8 + lr;
          float o[8];
          get8(u * 8 + lr, o);
          if (g.ep.bias) {
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] += bias[j];
          }
          if (g.ep.pre) store8_as(g.ep.pre, r * g.ep.ld_pre + c, g.ep.dtype, o);
          activate8(o, g.ep.activation);
          if (g.ep.add) {
            float w[8];
            if (add16) widen8(add[u], g.ep.add_dtype, w); else load8_as(g.ep.add, r * g.ep.ld_add + c, GD_DTYPE_FP32, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] += w[j];
          }
          store8_as(g.ep.out, r * g.ep.ld_out + c, g.ep.out_dtype, o);
        }
      };
      const auto release = [&](uint32_t buf) {       // this warp has read its part of the sum
        fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_peer(peer_address(smem_u32(&sum_empty[buf]), 0));
      };
      const uint32_t from = tmem + (quarter * 32u << 16) + half;
      if constexpr (CHAINED) {
        float v[128];
#pragma unroll
        for (uint32_t c = 0; c < 128; ++c) v[c] = 0.f;
        for (uint32_t k = 0; k < g.blocks_k; k += g.chain, ++chain) {
          const uint32_t buf = chain & 1u;
          if (!mbar_wait(&sum_full[buf], (chain / 2) & 1u, abort)) { good = false; break; }
          fence_after();
#pragma unroll
          for (uint32_t c = 0; c < 128; c += 16) {
            float w[16];
            tmem_load8(from + buf * 256u + c, w);
            tmem_load8(from + buf * 256u + c + 8, w + 8);
            tmem_ready();
#pragma unroll
            for (int j = 0; j < 16; ++j) v[c + j] += w[j];
          }
          release(buf);
        }
        if (!good) break;
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q) {
          fetch(q);
          put(v + 32 * q);
          finish(q);
        }
      } else {
        const uint32_t buf = chain & 1u;
        fetch(0);
        if (!mbar_wait(&sum_full[buf], (chain / 2) & 1u, abort)) { good = false; break; }
        fence_after();
        ++chain;
#pragma unroll 1
        for (uint32_t q = 0; q < 4; ++q) {
          if (q) fetch(q);
          float v[32];
          tmem_load32(from + buf * 256u + 32 * q, v);
          tmem_ready();
          if (q == 3) release(buf);
          put(v);
          finish(q);
        }
      }
    }
    if (!good) s_abort = 1;
  }
  if (!good && lane == 0) atomicExch(g.status, GD_ERR_DEVICE_TIMEOUT);
  __syncwarp();
  fence_before();
  cluster_arrive();                                  // neither CTA leaves while the other's products read its memory or its warps signal
  cluster_wait();
  if (warp == kPairWarps) tmem_free<2>(tmem, 512);
}

template <bool A_MN, bool B_MN, bool CHAINED>
cudaError_t launch_pair(const PairArgs& g, cudaStream_t stream) {
  auto kernel = product_pair_kernel<A_MN, B_MN, CHAINED>;
  static PerDeviceInt ready;
  int dev;
  if (!ready.get(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kPairBytes);
    if (e != cudaSuccess) return e;
    ready.set(dev, 1);
  }
  const uint32_t pairs = std::min<uint64_t>((uint64_t)g.tiles_r * g.tiles_c, (uint64_t)sm_count() / 2);
  return launch_dependent(kernel, dim3(2 * pairs), dim3(kPairThreads), kPairBytes, stream, g);
}
template <bool A_MN, bool B_MN>
cudaError_t launch_majors(const PairArgs& g, cudaStream_t stream) {
  return g.chain < g.blocks_k ? launch_pair<A_MN, B_MN, true>(g, stream) : launch_pair<A_MN, B_MN, false>(g, stream);
}

}  // namespace

cudaError_t launch_product_pair(const Product& p, cudaStream_t stream) {
  PairArgs g;
  std::memset(&g, 0, sizeof(g));
  if (!encode_operand(&g.a, p.a, p.ep.rows, p.depth, p.a.mn_major ? 64 : 128, p.bf16) ||
      !encode_operand(&g.b, p.b, p.ep.cols, p.depth, p.b.mn_major ? 64 : 128, p.bf16))
    return cudaErrorInvalidValue;
  g.ep = p.ep;
  g.status = p.status;
  g.blocks_k = (p.depth + kBlockK - 1) / kBlockK;
  g.chain = chain_blocks(p);
  g.desc = mma_desc(256, 256, p.bf16, p.a.mn_major, p.b.mn_major);
  g.tiles_r = (p.ep.rows + 255) / 256;
  g.tiles_c = (p.ep.cols + 255) / 256;
  if (p.a.mn_major) return p.b.mn_major ? launch_majors<true, true>(g, stream) : cudaErrorInvalidValue;   // (no call has A alone transposed)
  return p.b.mn_major ? launch_majors<false, true>(g, stream) : launch_majors<false, false>(g, stream);
}

}  // namespace gd
