// The product of the gated block: both projections, the activation and the product of the two in one kernel.
//
// A tile's accumulator holds the gate's columns beside the same columns of the other projection, so that an epilogue lane has both and nothing
// but the result (and z, where it is kept) leaves the SM.  x is read once for both.  The two shapes are those of the plain products:
//
// Pairs of CTAs, persistent, for many tiles: 256 rows x 128 outputs.  The pair's instruction takes B's first half from the leading CTA's shared
// memory and the second from the other's: one loads the gate's rows of W, the other the same rows of the other half.  Bound by the tensor
// cores.  A piece of 32 rows x 64 columns leaves through shared memory by the copy engine, three of them where z is kept.
//
// A tile of 64 outputs x 16 .. 128 rows per CTA, k split over a cluster, for few tiles: the outputs lie on the accumulator's lanes, the gate's 64
// and the others' 64, so that few rows waste nothing.  Bound by the bytes of W, read by as many SMs as there are.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "gd_gated.cuh"

namespace gd {
namespace {

// ---------------------------------------------------------------- pairs
constexpr uint32_t kPairWarps = 8, kPairThreads = (kPairWarps + 2) * 32;
constexpr uint32_t kHalfA = 128 * kBlockK * 2, kPairStage = 2 * kHalfA;      // a CTA's rows of x and its 128 rows of W
constexpr uint32_t kPieceBytes = 32 * 128;
constexpr uint32_t kGroup = 8;
constexpr uint32_t kOutputs = 128;                 // of a tile
template <bool PRE>
struct PairShape {
  static constexpr uint32_t kStages = PRE ? 4 : 5, kPieces = PRE ? 3 : 2;
  static constexpr uint32_t kBytes = kStages * kPairStage + kPairWarps * kPieces * kPieceBytes + 1024;
};
struct PairArgs {
  CUtensorMap x, w[2];
  CUtensorMap out, pre[2];                         // pieces (TILED)
  GatedEpilogue ep;
  int* status;
  uint32_t blocks_k, desc, tiles_r, tiles_c;
};

template <bool B_MN, bool PRE, bool TILED>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kPairThreads, 1) gated_pair_kernel(const __grid_constant__ PairArgs g) {
  constexpr uint32_t kStages = PairShape<PRE>::kStages, kPieces = PairShape<PRE>::kPieces;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t full[kStages], empty[kStages], sum_full[2], sum_empty[2];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  const uint32_t rank = cluster_rank(), pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
  const uint32_t tiles = g.tiles_r * g.tiles_c;
  if (tid == 0) {
    for (uint32_t s = 0; s < kStages; ++s) mbar_init(&full[s], 1u), mbar_init(&empty[s], 1u);
    for (uint32_t s = 0; s < 2; ++s) mbar_init(&sum_full[s], 1u), mbar_init(&sum_empty[s], 2 * kPairWarps);   // (the leader's: both CTAs' warps)
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (g.blocks_k) prefetch_map(&g.x), prefetch_map(&g.w[rank]);
  }
  if (warp == kPairWarps) tmem_alloc<2>(&s_tmem, 512);
  fence_before();
  cluster_arrive();                                // both CTAs' barriers exist before either signals the other's
  cluster_wait();
  fence_after();
  const uint32_t tmem = s_tmem;
  const volatile int* abort = &s_abort;
  bool good = true;
  pdl_wait();
  pdl_trigger();
  // tiles in groups of kGroup tile rows, within a group column by column: what the pairs read at one time stays in L2
  const auto place = [&](uint32_t t, uint32_t* r, uint32_t* c) {
    const uint32_t in_group = kGroup * g.tiles_c, group = t / in_group, rest = t % in_group, rows = min(kGroup, g.tiles_r - group * kGroup);
    *r = group * kGroup + rest % rows;
    *c = rest / rows;
  };

  if (warp == kPairWarps) {                        // copies: each CTA its rows of x and its half of W, all counted on the leader's barrier
    if (elect_one()) {
      uint32_t n = 0;
      for (uint32_t t = pair; good && t < tiles; t += pairs) {
        uint32_t tr, tc;
        place(t, &tr, &tc);
        const int32_t i0 = (int32_t)(tr * 256u + rank * 128u), j0 = (int32_t)(tc * kOutputs);
        for (uint32_t k = 0; k < g.blocks_k; ++k, ++n) {
          const uint32_t s = n % kStages;
          if (n >= kStages && !mbar_wait(&empty[s], (n / kStages + 1u) & 1u, abort)) { good = false; break; }
          unsigned char* at = smem + s * kPairStage;
          const uint32_t bar = peer_address(smem_u32(&full[s]), 0);
          const int32_t kc = (int32_t)(k * kBlockK);
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2 * kPairStage);
          tile_load_pair(at, &g.x, kc, i0, bar);
          if constexpr (B_MN) {
            tile_load_pair(at + kHalfA, &g.w[rank], j0, kc, bar);
            tile_load_pair(at + kHalfA + 8192, &g.w[rank], j0 + 64, kc, bar);
          } else {
            tile_load_pair(at + kHalfA, &g.w[rank], kc, j0, bar);
          }
        }
      }
      // every block has been used (in the ordinary case): what the CTA asked for has landed, and nothing will still arrive at its barriers
      const int none = 0;
      if (!good) s_abort = 1;
      for (uint32_t u = n > kStages ? n - kStages : 0u; u < n; ++u) {
        if (good) good = mbar_wait(&empty[u % kStages], (u / kStages) & 1u, abort);
        else if (rank == 0) (void)mbar_wait(&full[u % kStages], (u / kStages) & 1u, &none);
      }
    }
  } else if (warp == kPairWarps + 1) {             // products, issued by the leader for both
    if (rank == 0 && elect_one()) {
      uint32_t n = 0, turn = 0;
      for (uint32_t t = pair; good && t < tiles; t += pairs, ++turn) {
        const uint32_t buf = turn & 1u, sum = tmem + buf * 256u;
        if (turn >= 2 && !mbar_wait(&sum_empty[buf], (turn / 2 + 1u) & 1u, abort)) { good = false; break; }
        fence_after();
        for (uint32_t k = 0; k < g.blocks_k; ++k, ++n) {
          const uint32_t s = n % kStages;
          if (!mbar_wait(&full[s], (n / kStages) & 1u, abort)) { good = false; break; }
          fence_after();
          const uint32_t at = smem_u32(smem + s * kPairStage);
#pragma unroll
          for (uint32_t q = 0; q < kBlockK / 16; ++q) {
            const uint64_t a = operand_desc(at + q * 32u, 8192u);
            const uint64_t b = operand_desc(at + kHalfA + q * (B_MN ? 2048u : 32u), 8192u);
            mma<2>(sum, a, b, g.desc, k | q);
          }
          mma_commit_pair(&empty[s]);
        }
        if (good) mma_commit_pair(&sum_full[buf]);
      }
      if (!good) s_abort = 1;
    }
  } else {
    // warps w and w + 4 take the lanes of quarter w, 64 outputs each: the gate's columns and, 128 further on, the others
    const uint32_t quarter = warp & 3u, half = (warp >> 2) * 64u;
    unsigned char* pieces = smem + kStages * kPairStage + warp * kPieces * kPieceBytes;
    const GatedEpilogue& ep = g.ep;
    uint32_t turn = 0;
    for (uint32_t t = pair; good && t < tiles; t += pairs, ++turn) {
      uint32_t tr, tc;
      place(t, &tr, &tc);
      const uint32_t r0 = tr * 256u + rank * 128u + quarter * 32u, c0 = tc * kOutputs + half, buf = turn & 1u;
      const uint32_t from = tmem + (quarter * 32u << 16) + buf * 256u + half;
      // lane l holds the bias of outputs l and 32 + l; asked for before the sum is there
      float bias_g[2] = {0.f, 0.f}, bias_u[2] = {0.f, 0.f};
      if (ep.bias) {
#pragma unroll
        for (uint32_t p = 0; p < 2; ++p) {
          const uint32_t c = c0 + 32u * p + lane;
          if (c < ep.cols) bias_g[p] = load_as(ep.bias, c, ep.bias_dtype), bias_u[p] = load_as(ep.bias, (uint64_t)ep.cols + c, ep.bias_dtype);
        }
      }
      unsigned char* out = pieces + (PRE ? 0u : buf) * kPieceBytes;
      if constexpr (TILED) {                       // the pieces' place is free
        if (elect_one()) { if (PRE) stores_read<0>(); else stores_read<1>(); }
        __syncwarp();
      }
      good = mbar_wait(&sum_full[buf], (turn / 2) & 1u, abort);
      if (!good) break;
      fence_after();
#pragma unroll 1
      for (uint32_t p = 0; p < 2; ++p) {
        float zg[32], zu[32];
        tmem_load32(from + p * 32u, zg);
        tmem_load32(from + 128u + p * 32u, zu);
        tmem_ready();
        if (p == 1) {                              // this warp has read its part of the sum
          fence_before();
          __syncwarp();
          if (elect_one()) mbar_arrive_peer(peer_address(smem_u32(&sum_empty[buf]), 0));
        }
        if (ep.bias) {
          const float bg = p ? bias_g[1] : bias_g[0], bu = p ? bias_u[1] : bias_u[0];
#pragma unroll
          for (uint32_t j = 0; j < 32; ++j) zg[j] += __shfl_sync(0xFFFFFFFFu, bg, j), zu[j] += __shfl_sync(0xFFFFFFFFu, bu, j);
        }
        if constexpr (TILED) {
          const auto put = [&](unsigned char* piece, const float* v) {
#pragma unroll
            for (uint32_t j = 0; j < 4; ++j) *reinterpret_cast<uint4*>(piece + lane * 128u + ((p * 4u + j) ^ (lane & 7u)) * 16u) = narrow8(v + 8 * j, ep.dtype);
          };
          if constexpr (PRE) put(pieces + kPieceBytes, zg), put(pieces + 2 * kPieceBytes, zu);
          gate_all<32>(zg, zu, ep.activation);
          put(out, zg);
        } else {
          // any pitch: a row of 32 at a time, one column per lane, through one piece in fp32
          float* piece = reinterpret_cast<float*>(pieces);
          const auto put = [&](const float* v, void* to, uint64_t ld, uint64_t shift) {
            __syncwarp();
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j)
              *reinterpret_cast<float4*>(piece + lane * 32u + (j ^ (lane & 7u)) * 4u) = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
            __syncwarp();
            const uint32_t c = c0 + p * 32u + lane;
            if (c < ep.cols) {
#pragma unroll 8
              for (uint32_t r = 0; r < 32; ++r)
                if (r0 + r < ep.rows) store_as(to, (uint64_t)(r0 + r) * ld + shift + c, ep.dtype, piece[r * 32u + ((lane >> 2) ^ (r & 7u)) * 4u + (lane & 3u)]);
            }
          };
          if constexpr (PRE) put(zg, ep.pre, ep.ld_pre, 0), put(zu, ep.pre, ep.ld_pre, ep.cols);
          gate_all<32>(zg, zu, ep.activation);
          put(zg, ep.out, ep.ld_out, 0);
        }
      }
      if constexpr (TILED) {
        fence_async();
        __syncwarp();
        if (elect_one()) {
          if (r0 < ep.rows && c0 < ep.cols) {
            tile_store(&g.out, out, (int32_t)c0, (int32_t)r0);
            if constexpr (PRE) {
              tile_store(&g.pre[0], pieces + kPieceBytes, (int32_t)c0, (int32_t)r0);
              tile_store(&g.pre[1], pieces + 2 * kPieceBytes, (int32_t)c0, (int32_t)r0);
            }
          }
          stores_commit();
        }
      }
    }
    if constexpr (TILED) {
      if (elect_one()) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    if (!good) s_abort = 1;
  }
  if (!good) atomicExch(g.status, GD_ERR_DEVICE_TIMEOUT);
  __syncwarp();
  fence_before();
  cluster_arrive();                                // neither CTA leaves while the other's products read its memory or its warps signal
  cluster_wait();
  if (warp == kPairWarps) tmem_free<2>(tmem, 512);
}

template <bool B_MN, bool PRE, bool TILED>
cudaError_t launch_pair(const PairArgs& g, cudaStream_t stream) {
  auto kernel = gated_pair_kernel<B_MN, PRE, TILED>;
  static PerDeviceInt ready;
  int dev;
  if (!ready.get(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PairShape<PRE>::kBytes);
    if (e != cudaSuccess) return e;
    ready.set(dev, 1);
  }
  const uint32_t pairs = (uint32_t)std::min<uint64_t>((uint64_t)g.tiles_r * g.tiles_c, (uint64_t)sm_count() / 2);
  return launch_dependent(kernel, dim3(2 * pairs), dim3(kPairThreads), PairShape<PRE>::kBytes, stream, g);
}
cudaError_t launch_pairs(const GatedProduct& p, cudaStream_t stream) {
  PairArgs g;
  std::memset(&g, 0, sizeof(g));
  const GatedEpilogue& ep = p.ep;
  const bool b_mn = p.gate.mn_major, pre = ep.pre != nullptr, tiled = ep.vectors != 0;
  const uint32_t box = b_mn ? 64 : 128;
  if (!encode_operand(&g.x, p.x, ep.rows, p.depth, 128, p.bf16) || !encode_operand(&g.w[0], p.gate, ep.cols, p.depth, box, p.bf16) ||
      !encode_operand(&g.w[1], p.up, ep.cols, p.depth, box, p.bf16))
    return cudaErrorInvalidValue;
  g.ep = ep;
  g.status = p.status;
  g.blocks_k = (p.depth + kBlockK - 1) / kBlockK;
  g.desc = mma_desc(256, 256, p.bf16, false, b_mn);
  g.tiles_r = (ep.rows + 255) / 256;
  g.tiles_c = (ep.cols + kOutputs - 1) / kOutputs;
  if (tiled) {
    Epilogue like;
    std::memset(&like, 0, sizeof(like));
    like.rows = ep.rows, like.cols = ep.cols;
    if (!encode_piece(&g.out, ep.out, ep.ld_out, like, ep.cols, ep.dtype)) return cudaErrorInvalidValue;
    if (pre && (!encode_piece(&g.pre[0], ep.pre, ep.ld_pre, like, ep.cols, ep.dtype) ||
                !encode_piece(&g.pre[1], static_cast<uint16_t*>(ep.pre) + ep.cols, ep.ld_pre, like, ep.cols, ep.dtype)))
      return cudaErrorInvalidValue;
  }
  if (b_mn) {
    if (pre) return tiled ? launch_pair<true, true, true>(g, stream) : launch_pair<true, true, false>(g, stream);
    return tiled ? launch_pair<true, false, true>(g, stream) : launch_pair<true, false, false>(g, stream);
  }
  if (pre) return tiled ? launch_pair<false, true, true>(g, stream) : launch_pair<false, true, false>(g, stream);
  return tiled ? launch_pair<false, false, true>(g, stream) : launch_pair<false, false, false>(g, stream);
}

// ---------------------------------------------------------------- few tiles
constexpr uint32_t kSumWarps = 8, kThreadsSplit = (kSumWarps + 2) * 32;      // + one warp that asks for copies, one that issues products
constexpr uint32_t kTileA = 128 * kBlockK * 2;       // of W: 64 outputs of either half
constexpr uint32_t kTileOutputs = 64, kPitch = 132;  // partial tile: a row of 128 lanes per row of x
constexpr uint32_t kMostStages = 10;
template <int BN>
struct SplitShape {
  static constexpr uint32_t kStage = kTileA + BN * kBlockK * 2;
  static constexpr uint32_t kPartial = BN * kPitch * 4;        // takes the blocks' place
};
struct SplitArgs {
  CUtensorMap w[2], x;
  GatedEpilogue ep;
  int* status;
  uint32_t blocks_k, tiles_i, desc, stages;
};

__device__ __forceinline__ void finish_gated8(const GatedEpilogue& e, uint32_t r, uint32_t c, float (&g)[8], float (&u)[8]) {
  if (e.vectors) {
    if (c >= e.cols) return;
    if (e.bias) {
      float b[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = load_as(e.bias, c + j, e.bias_dtype);
#pragma unroll
      for (int j = 0; j < 8; ++j) g[j] += b[j];
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = load_as(e.bias, (uint64_t)e.cols + c + j, e.bias_dtype);
#pragma unroll
      for (int j = 0; j < 8; ++j) u[j] += b[j];
    }
    if (e.pre) {
      store8_as(e.pre, (uint64_t)r * e.ld_pre + c, e.dtype, g);
      store8_as(e.pre, (uint64_t)r * e.ld_pre + e.cols + c, e.dtype, u);
    }
    gate_all<8>(g, u, e.activation);
    store8_as(e.out, (uint64_t)r * e.ld_out + c, e.dtype, g);
    return;
  }
#pragma unroll
  for (uint32_t j = 0; j < 8; ++j) {
    if (c + j >= e.cols) break;
    float a = g[j], b = u[j];
    if (e.bias) a += load_as(e.bias, c + j, e.bias_dtype), b += load_as(e.bias, (uint64_t)e.cols + c + j, e.bias_dtype);
    if (e.pre) {
      store_as(e.pre, (uint64_t)r * e.ld_pre + c + j, e.dtype, a);
      store_as(e.pre, (uint64_t)r * e.ld_pre + e.cols + c + j, e.dtype, b);
    }
    store_as(e.out, (uint64_t)r * e.ld_out + c + j, e.dtype, activate(a, e.activation) * b);
  }
}

template <bool W_MN, int BN, int SPLITS>
__global__ void __launch_bounds__(kThreadsSplit, 2) gated_split_kernel(const __grid_constant__ SplitArgs g) {
  using S = SplitShape<BN>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t full[kMostStages], empty[kMostStages], sum_full;
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  constexpr uint32_t kColumns = BN < 32 ? 32 : BN;
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  const uint32_t rank = SPLITS > 1 ? cluster_rank() : 0u, tile = blockIdx.x / SPLITS;
  const uint32_t i0 = tile % g.tiles_i * kTileOutputs, j0 = tile / g.tiles_i * BN;
  const uint32_t k0 = (uint64_t)g.blocks_k * rank / SPLITS, k1 = (uint64_t)g.blocks_k * (rank + 1) / SPLITS;
  if (tid == 0) {
    for (uint32_t s = 0; s < kMostStages; ++s) mbar_init(&full[s], 1u), mbar_init(&empty[s], 1u);
    mbar_init(&sum_full, 1u);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (g.blocks_k) prefetch_map(&g.w[0]), prefetch_map(&g.w[1]), prefetch_map(&g.x);
  }
  if (warp == kSumWarps) tmem_alloc<1>(&s_tmem, kColumns);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  const volatile int* abort = &s_abort;
  pdl_wait();
  pdl_trigger();

  float* part = reinterpret_cast<float*>(smem);
  constexpr uint32_t kHalf = BN / 2;
  float v[kHalf];
  bool good = true;
  if (warp == kSumWarps) {                           // copies
    if (elect_one()) {
      uint32_t issued = 0, s = 0, parity = 1;        // (a fresh barrier reads as "the phase of parity 1 is over")
      for (uint32_t k = k0; k < k1; ++k, ++issued) {
        if (!mbar_wait(&empty[s], parity, abort)) { good = false; break; }
        unsigned char* at = smem + s * S::kStage;
        const int32_t kc = (int32_t)(k * kBlockK);
        mbar_arrive_expect_tx(&full[s], S::kStage);
#pragma unroll
        for (uint32_t h = 0; h < 2; ++h) {
          if constexpr (W_MN) tile_load(at + h * 8192u, &g.w[h], (int32_t)i0, kc, &full[s]);
          else tile_load(at + h * 8192u, &g.w[h], kc, (int32_t)i0, &full[s]);
        }
        tile_load(at + kTileA, &g.x, kc, (int32_t)j0, &full[s]);
        if (++s == g.stages) s = 0, parity ^= 1u;
      }
      if (!good) {                                   // a wait ran out: let the copies in flight land before the CTA may end
        s_abort = 1;
        const int none = 0;
        for (uint32_t n = issued > g.stages ? issued - g.stages : 0u; n < issued; ++n)
          (void)mbar_wait(&full[n % g.stages], (n / g.stages) & 1u, &none);
      }
    }
  } else if (warp == kSumWarps + 1) {                // products
    if (elect_one() && k0 < k1) {
      uint32_t s = 0, parity = 0;
      for (uint32_t k = k0; k < k1; ++k) {
        if (!mbar_wait(&full[s], parity, abort)) { good = false; break; }
        fence_after();
        const uint32_t at = smem_u32(smem + s * S::kStage);
#pragma unroll
        for (uint32_t q = 0; q < kBlockK / 16; ++q) {
          const uint64_t a = operand_desc(at + q * (W_MN ? 2048u : 32u), 8192u);
          const uint64_t b = operand_desc(at + kTileA + q * 32u, 8192u);
          mma<1>(tmem, a, b, g.desc, (k - k0) | q);
        }
        mma_commit(&empty[s]);
        if (++s == g.stages) s = 0, parity ^= 1u;
      }
      if (good) mma_commit(&sum_full);
      else s_abort = 1;
    }
  } else {
    // warps w and w + 4 take the lanes of quarter w, half of the rows each
    const uint32_t quarter = warp & 3u, c0 = (warp >> 2) * kHalf;
#pragma unroll
    for (uint32_t c = 0; c < kHalf; ++c) v[c] = 0.f;
    if (k0 < k1) {
      good = mbar_wait(&sum_full, 0u, abort);
      if (good) {
        fence_after();
#pragma unroll
        for (uint32_t c = 0; c < kHalf; c += 8) tmem_load8(tmem + (quarter * 32u << 16) + c0 + c, v + c);
        tmem_ready();
        fence_before();
      } else {
        s_abort = 1;
      }
    }
  }
  if (!good) atomicExch(g.status, GD_ERR_DEVICE_TIMEOUT);
  __syncthreads();                                   // every product is done and every copy has landed: the blocks' place is free
  if (warp < kSumWarps) {
    const uint32_t c0 = (warp >> 2) * kHalf, i = (warp & 3u) * 32u + lane;
#pragma unroll
    for (uint32_t c = 0; c < kHalf; ++c) part[(c0 + c) * kPitch + i] = v[c];
  }
  if constexpr (SPLITS > 1) {
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
  // this CTA's rows of the tile, eight outputs a thread; the parts in rank order
  constexpr uint32_t kMyRows = BN / SPLITS, kVecs = kTileOutputs / 8u;
  for (uint32_t t = tid; t < kMyRows * kVecs; t += kThreadsSplit) {
    const uint32_t r = rank * kMyRows + t / kVecs, c = t % kVecs * 8u;
    if (j0 + r >= g.ep.rows) continue;
    const float* at = part + r * kPitch + c;
    float z[2][8];
#pragma unroll
    for (uint32_t h = 0; h < 2; ++h) {
#pragma unroll
      for (uint32_t q = 0; q < SPLITS; ++q) {
        float4 a, b;
        if constexpr (SPLITS > 1) {
          const uint32_t peer = peer_address(smem_u32(at + h * kTileOutputs), q);
          a = peer_load4(peer), b = peer_load4(peer + 16);
        } else {
          a = *reinterpret_cast<const float4*>(at + h * kTileOutputs), b = *reinterpret_cast<const float4*>(at + h * kTileOutputs + 4);
        }
        const float w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int j = 0; j < 8; ++j) z[h][j] = q == 0 ? w[j] : z[h][j] + w[j];
      }
    }
    finish_gated8(g.ep, j0 + r, i0 + c, z[0], z[1]);
  }
  if constexpr (SPLITS > 1) {
    cluster_arrive();                                // the others may still be reading this CTA's partial tile
    cluster_wait();
  } else {
    __syncthreads();
  }
  if (warp == kSumWarps) tmem_free<1>(tmem, kColumns);
}

template <bool W_MN, int BN, int SPLITS>
cudaError_t launch_shape(const SplitArgs& g, uint32_t tiles, cudaStream_t stream) {
  auto kernel = gated_split_kernel<W_MN, BN, SPLITS>;
  static PerDeviceInt ready;
  int dev;
  if (!ready.get(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 201 * 1024);
    if (e != cudaSuccess) return e;
    ready.set(dev, 1);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(tiles * SPLITS);
  cfg.blockDim = dim3(kThreadsSplit);
  cfg.dynamicSmemBytes = std::max(g.stages * SplitShape<BN>::kStage, SplitShape<BN>::kPartial) + 1024;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = SPLITS;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = SPLITS > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, g);
}
template <bool W_MN, int BN>
cudaError_t launch_splits(uint32_t splits, const SplitArgs& g, uint32_t tiles, cudaStream_t stream) {
  switch (splits) {
    case 1: return launch_shape<W_MN, BN, 1>(g, tiles, stream);
    case 2: return launch_shape<W_MN, BN, 2>(g, tiles, stream);
    case 4: return launch_shape<W_MN, BN, 4>(g, tiles, stream);
    default: return launch_shape<W_MN, BN, 8>(g, tiles, stream);
  }
}
template <bool W_MN>
cudaError_t launch_bn(uint32_t bn, uint32_t splits, const SplitArgs& g, uint32_t tiles, cudaStream_t stream) {
  switch (bn) {
    case 16: return launch_splits<W_MN, 16>(splits, g, tiles, stream);
    case 32: return launch_splits<W_MN, 32>(splits, g, tiles, stream);
    case 64: return launch_splits<W_MN, 64>(splits, g, tiles, stream);
    default: return launch_splits<W_MN, 128>(splits, g, tiles, stream);
  }
}

struct Choice {
  uint32_t bn, splits;        // of the smallest estimated time among the tiles of few
  double cost;                // in cycles of an SM
};
// The estimate of the plain product's tiles (gd_product_split.cu), where a tile is 64 outputs of either half.
Choice choose_split(const GatedProduct& p) {
  const uint32_t sms = (uint32_t)sm_count(), blocks_k = (p.depth + kBlockK - 1) / kBlockK;
  Choice best{128, 1, 1e300};
  for (uint32_t bn = 16; bn <= 128; bn *= 2) {
    const uint32_t bytes = kTileA + bn * kBlockK * 2;
    const double tiles = std::ceil(p.ep.cols / (double)kTileOutputs) * std::ceil(p.ep.rows / (double)bn);
    for (uint32_t splits = 1; splits <= 8; splits *= 2) {
      if (splits > 1 && blocks_k < 2 * splits) break;
      const double ctas = tiles * splits, share = ctas <= sms ? 1.0 : 2.0, blocks = std::ceil(blocks_k / (double)splits);
      const double block = share * std::max(2.0 * bn, bytes / 72.0);
      const double exchange = splits == 1 ? 0.0 : splits == 2 ? 2200.0 : splits == 4 ? 3750.0 : 7400.0;
      const double cost = 2600.0 + std::ceil(ctas / (share * sms)) * (blocks * block + share * 33.0 * bn + 3750.0 + exchange);
      if (cost < best.cost) best = Choice{bn, splits, cost};
    }
  }
  return best;
}
double cost_pairs(const GatedProduct& p) {
  const double tiles = std::ceil(p.ep.rows / 256.0) * std::ceil(p.ep.cols / (double)kOutputs), blocks_k = std::ceil(p.depth / (double)kBlockK);
  return 12600.0 + std::ceil(tiles / (sm_count() / 2)) * std::max(600.0 * blocks_k, 9000.0);
}

cudaError_t launch_split(const GatedProduct& p, const Choice& c, cudaStream_t stream) {
  SplitArgs g;
  std::memset(&g, 0, sizeof(g));
  const bool w_mn = p.gate.mn_major;
  if (p.depth && (!encode_operand(&g.w[0], p.gate, p.ep.cols, p.depth, 64, p.bf16) || !encode_operand(&g.w[1], p.up, p.ep.cols, p.depth, 64, p.bf16) ||
                  !encode_operand(&g.x, p.x, p.ep.rows, p.depth, c.bn, p.bf16)))
    return cudaErrorInvalidValue;
  g.ep = p.ep;
  g.status = p.status;
  g.blocks_k = (p.depth + kBlockK - 1) / kBlockK;
  g.tiles_i = (p.ep.cols + kTileOutputs - 1) / kTileOutputs;
  g.desc = mma_desc(128, c.bn, p.bf16, w_mn, false);
  const uint64_t tiles = (uint64_t)g.tiles_i * ((p.ep.rows + c.bn - 1) / c.bn);
  if (tiles * c.splits > 0x7FFFFFFFull) return cudaErrorInvalidValue;
  // copies under way: what the CTAs of an SM have room for, with one of them or two
  g.stages = std::min((tiles * c.splits <= (uint64_t)sm_count() ? 200u : 98u) * 1024u / (kTileA + c.bn * kBlockK * 2), kMostStages);
  return w_mn ? launch_bn<true>(c.bn, c.splits, g, (uint32_t)tiles, stream) : launch_bn<false>(c.bn, c.splits, g, (uint32_t)tiles, stream);
}

}  // namespace

cudaError_t launch_gated_product(const GatedProduct& p, cudaStream_t stream) {
  if (p.ep.rows == 0 || p.ep.cols == 0) return cudaSuccess;
  const Choice split = choose_split(p);
  ProfileScope ps(stream, PT_GATED);
  const cudaError_t e = p.depth && cost_pairs(p) < split.cost ? launch_pairs(p, stream) : launch_split(p, split, stream);
  if (e == cudaSuccess) note_launches(1);
  return e;
}

}  // namespace gd
