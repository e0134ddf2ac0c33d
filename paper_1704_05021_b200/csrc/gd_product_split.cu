// The product for outputs of few tiles: one tile of 128 x BN per CTA, the contraction split over a cluster of 1 .. 8 CTAs.
//
// What bounds these calls is not arithmetic but how many SMs take part and how many bytes each keeps in flight: one row through a
// 4096 x 4096 layer is 33 MB of weights and next to no products.  So the longer side of the output lies on the tile's
// 128 accumulator lanes and the shorter one on its BN columns (the output is then written transposed, which costs nothing: the lanes of
// a warp are neighbours in memory), BN shrinks with the shorter side, and where there are fewer tiles than SMs the CTAs of
// a cluster take a part of k each.  They put their partial tiles into shared memory and every one sums, in rank order, the slice of
// rows it then finishes and stores: no workspace, no atomics, the same bits every time.  Where even eight CTAs per tile leave SMs idle over
// a long k, up to 16 such clusters take a part each and a second launch joins their sums (in workspace, in order).  Two CTAs share an SM
// where there are enough, so one's copies run under the other's epilogue.
//
// Measured (one B200, passes back to back on the device): 1 x 4096 x 4096 8.7 us (5.2 of weights), 512 x 512 x 512 3.7 us,
// 80 x 4096 x 784 5.0 us, 256 x 256 x 8192 8.8 us (24.6 without the split).
#include <algorithm>
#include <cmath>
#include <cstring>

#include "gd_mma.cuh"

namespace gd {
namespace {

constexpr uint32_t kSumWarps = 8, kThreadsSplit = (kSumWarps + 2) * 32;      // + one warp that asks for copies, one that issues products
constexpr uint32_t kTileA = 128 * kBlockK * 2;      // bytes of A's block

template <bool B_MN, int BN>
struct SplitShape {
  static constexpr uint32_t kTileB = (B_MN && BN < 64 ? 64 : BN) * kBlockK * 2;
  static constexpr uint32_t kStage = kTileA + kTileB;
  static constexpr uint32_t kPitchLanes = 132;      // partial tile, one row per column of D (output written transposed)
  static constexpr uint32_t kPitchCols = BN + 4;    // partial tile, one row per lane of D
  static constexpr uint32_t kPartial = (128 * kPitchCols > BN * kPitchLanes ? 128 * kPitchCols : BN * kPitchLanes) * 4;   // takes the blocks' place
};
// Copies a CTA keeps under way.  A block takes about 2500 cycles to arrive, so the more the better, up to what the CTAs of an SM have room
// for: with two of them 100 KB each, with one (no more CTAs than SMs) 200 KB.  1536 x 1024 x 4096, 96 CTAs of 64 blocks: 3 blocks deep
// 28.6 us, 6 deep 17.6.
constexpr uint32_t kMaxStages = 10;
uint32_t stages_for(uint32_t stage_bytes, bool alone) { return std::min((alone ? 200u : 98u) * 1024u / stage_bytes, kMaxStages); }

struct SplitArgs {
  CUtensorMap a, b;
  Epilogue ep;
  int* status;
  uint32_t blocks_k, tiles_i, desc;
  uint32_t chain;          // k blocks the tensor cores sum before the sum is joined to the others in fp32 registers
  uint32_t stages;         // blocks the shared memory holds
  uint32_t tiles, outer;   // outer > 1: the results are partial sums, part o of them partial_step elements on
  uint64_t partial_step;
  uint32_t transposed;     // D's lanes are the output's columns
  uint32_t beside;
};

template <bool A_MN, bool B_MN, int BN, int SPLITS>
__global__ void __launch_bounds__(kThreadsSplit, 2) product_split_kernel(const __grid_constant__ SplitArgs g) {
  using S = SplitShape<B_MN, BN>;
  extern __shared__ unsigned char smem_raw[];
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], sum_full[2], sum_empty[2];
  __shared__ uint32_t s_tmem;
  __shared__ int s_abort;
  unsigned char* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  constexpr uint32_t kColumns = BN < 32 ? 32 : 2 * BN;      // two accumulators
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  const uint32_t rank = SPLITS > 1 ? cluster_rank() : 0u, place = blockIdx.x / SPLITS, part_o = place / g.tiles, tile = place - part_o * g.tiles;
  const uint32_t i0 = tile % g.tiles_i * 128u, j0 = tile / g.tiles_i * BN;
  const uint32_t parts = g.outer * SPLITS, mine = part_o * SPLITS + rank;
  const uint32_t k0 = (uint64_t)g.blocks_k * mine / parts, k1 = (uint64_t)g.blocks_k * (mine + 1) / parts;
  if (tid == 0) {
    for (uint32_t s = 0; s < kMaxStages; ++s) mbar_init(&full[s], 1u), mbar_init(&empty[s], 1u);
    for (uint32_t s = 0; s < 2; ++s) mbar_init(&sum_full[s], 1u), mbar_init(&sum_empty[s], kSumWarps);
    s_abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    if (g.blocks_k) prefetch_map(&g.a), prefetch_map(&g.b);
  }
  if (warp == kSumWarps) tmem_alloc<1>(&s_tmem, kColumns);
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = s_tmem;
  const volatile int* abort = &s_abort;
  if (!g.beside) pdl_wait();                         // (the other product's CTAs are past theirs: all have triggered)
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
        mbar_arrive_expect_tx(&full[s], S::kStage);
        if constexpr (A_MN) {
          tile_load(at, &g.a, (int32_t)i0, (int32_t)(k * kBlockK), &full[s]);
          tile_load(at + 8192, &g.a, (int32_t)i0 + 64, (int32_t)(k * kBlockK), &full[s]);
        } else {
          tile_load(at, &g.a, (int32_t)(k * kBlockK), (int32_t)i0, &full[s]);
        }
        if constexpr (B_MN) {
#pragma unroll
          for (uint32_t c = 0; c < S::kTileB / 8192u; ++c)
            tile_load(at + kTileA + c * 8192u, &g.b, (int32_t)(j0 + c * 64u), (int32_t)(k * kBlockK), &full[s]);
        } else {
          tile_load(at + kTileA, &g.b, (int32_t)(k * kBlockK), (int32_t)j0, &full[s]);
        }
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
    if (elect_one()) {
      uint32_t s = 0, parity = 0, chain = 0;
      for (uint32_t k = k0; good && k < k1; ++chain) {
        const uint32_t end = min(k + g.chain, k1), buf = chain & 1u, sum = tmem + buf * BN;
        if (chain >= 2 && !mbar_wait(&sum_empty[buf], (chain / 2 + 1u) & 1u, abort)) { good = false; break; }
        fence_after();
        for (const uint32_t first = k; k < end; ++k) {
          if (!mbar_wait(&full[s], parity, abort)) { good = false; break; }
          fence_after();
          const uint32_t at = smem_u32(smem + s * S::kStage);
#pragma unroll
          for (uint32_t q = 0; q < kBlockK / 16; ++q) {
            const uint64_t a = operand_desc(at + q * (A_MN ? 2048u : 32u), 8192u);
            const uint64_t b = operand_desc(at + kTileA + q * (B_MN ? 2048u : 32u), 8192u);
            mma<1>(sum, a, b, g.desc, (k - first) | q);
          }
          mma_commit(&empty[s]);
          if (++s == g.stages) s = 0, parity ^= 1u;
        }
        if (good) mma_commit(&sum_full[buf]);
      }
      if (!good) s_abort = 1;
    }
  } else {
    // the chains' sums, joined in registers: warps w and w + 4 take the lanes of quarter w, half of the columns each
    const uint32_t quarter = warp & 3u, c0 = (warp >> 2) * kHalf, i = quarter * 32u + lane;
#pragma unroll
    for (uint32_t c = 0; c < kHalf; ++c) v[c] = 0.f;
    uint32_t chain = 0;
    for (uint32_t k = k0; k < k1; k += g.chain, ++chain) {
      const uint32_t buf = chain & 1u;
      if (!mbar_wait(&sum_full[buf], (chain / 2) & 1u, abort)) { good = false; break; }
      fence_after();
#pragma unroll
      for (uint32_t c = 0; c < kHalf; c += 8) {
        float t[8];
        tmem_load8(tmem + (quarter * 32u << 16) + buf * BN + c0 + c, t);
        tmem_ready();
#pragma unroll
        for (int j = 0; j < 8; ++j) v[c + j] += t[j];
      }
      fence_before();
      if (lane == 0) mbar_arrive(&sum_empty[buf]);
    }
    if (!good) s_abort = 1;
  }
  if (!good) atomicExch(g.status, GD_ERR_DEVICE_TIMEOUT);
  __syncthreads();                                   // every product is done and every copy has landed: the blocks' place is free
  if (warp < kSumWarps) {
    const uint32_t c0 = (warp >> 2) * kHalf, i = (warp & 3u) * 32u + lane;
    if (g.transposed) {
#pragma unroll
      for (uint32_t c = 0; c < kHalf; ++c) part[(c0 + c) * S::kPitchLanes + i] = v[c];
    } else {
#pragma unroll
      for (uint32_t c = 0; c < kHalf; c += 4)
        *reinterpret_cast<float4*>(part + i * S::kPitchCols + c0 + c) = make_float4(v[c], v[c + 1], v[c + 2], v[c + 3]);
    }
  }
  if constexpr (SPLITS > 1) {
    cluster_arrive();
    cluster_wait();
  } else {
    __syncthreads();
  }
  // this CTA's rows of the output tile
  const uint32_t rows = (g.transposed ? BN : 128u) / SPLITS, vecs = (g.transposed ? 128u : BN) / 8u;
  const uint32_t pitch = g.transposed ? S::kPitchLanes : S::kPitchCols;
  const uint32_t out_r = (g.transposed ? j0 : i0) + rank * rows, out_c = g.transposed ? i0 : j0;
  Epilogue ep = g.ep;
  if (g.outer > 1) ep.out = static_cast<float*>(ep.out) + part_o * g.partial_step;
  if (ep.vectors) {
    for (uint32_t t = tid; t < rows * vecs; t += kThreadsSplit) {
      const uint32_t r = t / vecs, c = t % vecs * 8u;
      const float* at = part + (rank * rows + r) * pitch + c;
      float v[8];
      if constexpr (SPLITS > 1) {
        const uint32_t address = smem_u32(at);
#pragma unroll
        for (uint32_t q = 0; q < SPLITS; ++q) {
          const uint32_t peer = peer_address(address, q);
          const float4 x = peer_load4(peer), y = peer_load4(peer + 16);
          const float w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
          for (int j = 0; j < 8; ++j) v[j] = q == 0 ? w[j] : v[j] + w[j];
        }
      } else {
        const float4 x = *reinterpret_cast<const float4*>(at), y = *reinterpret_cast<const float4*>(at + 4);
        v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w, v[4] = y.x, v[5] = y.y, v[6] = y.z, v[7] = y.w;
      }
      finish8(ep, out_r + r, out_c + c, v);
    }
  } else if (ep.pairs) {
    // rows that start at a multiple of 4 bytes: two columns per thread, up to eight rows of them at a time
    const uint32_t cols = vecs * 4u, group = rows < 8u ? rows : 8u;
    for (uint32_t t = tid; t < rows / group * cols; t += kThreadsSplit) {
      const uint32_t r = t / cols * group, c = t % cols * 2u;
      const float* at = part + (rank * rows + r) * pitch + c;
      if (out_c + c >= ep.cols || out_r + r >= ep.rows) continue;
      const float b0 = ep.bias ? load_as(ep.bias, out_c + c, ep.bias_dtype) : 0.f;
      const float b1 = ep.bias && out_c + c + 1 < ep.cols ? load_as(ep.bias, out_c + c + 1, ep.bias_dtype) : 0.f;
      float v[8], y[8];
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u) {
        if (u >= group) continue;
        float2 f;
        if constexpr (SPLITS > 1) {
          const uint32_t address = smem_u32(at + u * pitch);
#pragma unroll
          for (uint32_t q = 0; q < SPLITS; ++q) {
            const float2 w = peer_load2(peer_address(address, q));
            f = q == 0 ? w : make_float2(f.x + w.x, f.y + w.y);
          }
        } else {
          f = *reinterpret_cast<const float2*>(at + u * pitch);
        }
        v[u] = f.x + b0, y[u] = f.y + b1;
      }
      finish_columns(ep, out_r + r, out_c + c, v, y, group);
    }
  } else {
    // rows that start anywhere: a column per thread, up to eight rows of it at a time
    const uint32_t cols = vecs * 8u, group = rows < 8u ? rows : 8u;
    for (uint32_t t = tid; t < rows / group * cols; t += kThreadsSplit) {
      const uint32_t r = t / cols * group, c = t % cols;
      const float* at = part + (rank * rows + r) * pitch + c;
      if (out_c + c >= ep.cols || out_r + r >= ep.rows) continue;
      const float bias = ep.bias ? load_as(ep.bias, out_c + c, ep.bias_dtype) : 0.f;
      float v[8];
#pragma unroll
      for (uint32_t u = 0; u < 8; ++u) {
        if (u >= group) continue;
        if constexpr (SPLITS > 1) {
          const uint32_t address = smem_u32(at + u * pitch);
#pragma unroll
          for (uint32_t q = 0; q < SPLITS; ++q) {
            const float w = peer_load1(peer_address(address, q));
            v[u] = q == 0 ? w : v[u] + w;
          }
        } else {
          v[u] = at[u * pitch];
        }
        v[u] += bias;
      }
      finish_column(ep, out_r + r, out_c + c, v, group);
    }
  }
  if constexpr (SPLITS > 1) {
    cluster_arrive();                                // the others may still be reading this CTA's partial tile
    cluster_wait();
  } else {
    __syncthreads();
  }
  if (warp == kSumWarps) tmem_free<1>(tmem, kColumns);
  if (g.beside) pdl_wait();
}

template <bool A_MN, bool B_MN, int BN, int SPLITS>
cudaError_t launch_shape(const SplitArgs& g, uint32_t tiles, cudaStream_t stream) {
  const uint32_t bytes = std::max(g.stages * SplitShape<B_MN, BN>::kStage, SplitShape<B_MN, BN>::kPartial) + 1024;       // + alignment of the blocks
  auto kernel = product_split_kernel<A_MN, B_MN, BN, SPLITS>;
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
  cfg.dynamicSmemBytes = bytes;
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
template <bool A_MN, bool B_MN, int BN>
cudaError_t launch_splits(uint32_t splits, const SplitArgs& g, uint32_t tiles, cudaStream_t stream) {
  switch (splits) {
    case 1: return launch_shape<A_MN, B_MN, BN, 1>(g, tiles, stream);
    case 2: return launch_shape<A_MN, B_MN, BN, 2>(g, tiles, stream);
    case 4: return launch_shape<A_MN, B_MN, BN, 4>(g, tiles, stream);
    default: return launch_shape<A_MN, B_MN, BN, 8>(g, tiles, stream);
  }
}
template <bool A_MN, bool B_MN>
cudaError_t launch_bn(uint32_t bn, uint32_t splits, const SplitArgs& g, uint32_t tiles, cudaStream_t stream) {
  switch (bn) {
    case 16: return launch_splits<A_MN, B_MN, 16>(splits, g, tiles, stream);
    case 32: return launch_splits<A_MN, B_MN, 32>(splits, g, tiles, stream);
    case 64: return launch_splits<A_MN, B_MN, 64>(splits, g, tiles, stream);
    default: return launch_splits<A_MN, B_MN, 128>(splits, g, tiles, stream);
  }
}

uint32_t tile_bytes(uint32_t bn, bool j_mn) { return kTileA + (j_mn && bn < 64 ? 64 : bn) * kBlockK * 2; }
// out = epilogue of the sum of `outer` partial sums, in order.  A thread takes eight neighbours of a row.
__global__ void __launch_bounds__(256) join_kernel(const __grid_constant__ Epilogue ep, const float* partial, uint64_t step, uint32_t ld, uint32_t outer) {
  pdl_wait();
  pdl_trigger();
  const uint64_t t = (uint64_t)blockIdx.x * 256u + threadIdx.x;
  const uint32_t vecs = ld / 8u, r = (uint32_t)(t / vecs), c = (uint32_t)(t % vecs) * 8u;
  if (r >= ep.rows) return;
  float v[8] = {};
  for (uint32_t o = 0; o < outer; ++o) {
    float w[8];
    load8_as(partial + o * step, (uint64_t)r * ld + c, GD_DTYPE_FP32, w);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] += w[j];
  }
  finish8(ep, r, c, v);
}

// The tile shape and split with the smallest estimated time, in cycles of an SM.  A block takes the longer of its products (2 BN cycles)
// and its copies (72 bytes per cycle) for as many CTAs as share the SM; a CTA costs its start, its first block's latency and its
// epilogue besides, a split the exchange of the partial tiles.  The constants are a least-squares fit of the logarithms of 500 measured times
// (20 shapes, all tiles and splits; within 15 % in the middle); the choice it makes is the fastest or within 10 % of it on all but
// one of the shapes (10 outputs' gradient of 80 x 4096: 5.7 against 4.7 us).
SplitChoice choose(uint32_t rows, uint32_t cols, uint32_t blocks_k, bool a_mn, bool b_mn, bool can_join, bool followed) {
  const uint32_t sms = (uint32_t)sm_count();
  SplitChoice best{false, 128, 1, 1, 1e300};
  for (int t = 0; t < 2; ++t) {
    const uint32_t ei = t ? cols : rows, ej = t ? rows : cols;
    const bool j_mn = t ? a_mn : b_mn;
    for (uint32_t bn = 16; bn <= 128; bn *= 2) {
      const uint32_t bytes = tile_bytes(bn, j_mn);
      const double tiles = std::ceil(ei / 128.0) * std::ceil(ej / (double)bn);
      for (uint32_t splits = 1; splits <= 8; splits *= 2) {
        if (splits > 1 && blocks_k < 2 * splits) break;
        // outputs of so few tiles that eight CTAs each leave SMs idle over a long k: the join is a launch and a trip through L2
        for (uint32_t outer = 1; outer <= 16; outer *= 2) {
          if (outer > 1 && (!can_join || splits < 8 || blocks_k < 32 * outer || (uint64_t)outer * rows * ((cols + 7) / 8 * 8) * 4 > kPartialBytes)) break;
          const double ctas = tiles * splits * outer, share = ctas <= sms ? 1.0 : 2.0, blocks = std::ceil(blocks_k / (double)(splits * outer));
          const double block = share * std::max(2.0 * bn, bytes / 72.0);
          const double exchange = splits == 1 ? 0.0 : splits == 2 ? 2200.0 : splits == 4 ? 3750.0 : 7400.0;
          const double cost =
              2600.0 + (followed ? std::max(1.0, ctas / (share * sms)) : std::ceil(ctas / (share * sms))) * (blocks * block + share * 33.0 * bn + 3750.0 + exchange) + (outer > 1 ? 6000.0 : 0.0);
          if (cost < best.cost) best = SplitChoice{t != 0, bn, splits, outer, cost};
        }
      }
    }
  }
  return best;
}

}  // namespace

SplitChoice choose_product_split(const Product& p) {
  return choose(p.ep.rows, p.ep.cols, (p.depth + kBlockK - 1) / kBlockK, p.a.mn_major, p.b.mn_major, p.partial != nullptr, p.followed);
}

cudaError_t launch_product_split(const Product& p, const SplitChoice& c, cudaStream_t stream) {
  const uint32_t blocks_k = (p.depth + kBlockK - 1) / kBlockK;
  const Operand& oi = c.transposed ? p.b : p.a;
  const Operand& oj = c.transposed ? p.a : p.b;
  const uint32_t ei = c.transposed ? p.ep.cols : p.ep.rows, ej = c.transposed ? p.ep.rows : p.ep.cols;
  SplitArgs g;
  std::memset(&g, 0, sizeof(g));
  if (p.depth && (!encode_operand(&g.a, oi, ei, p.depth, oi.mn_major ? 64 : 128, p.bf16) ||
                  !encode_operand(&g.b, oj, ej, p.depth, oj.mn_major ? 64 : c.bn, p.bf16)))
    return cudaErrorInvalidValue;
  g.ep = p.ep;
  g.status = p.status;
  g.beside = p.beside;
  g.blocks_k = blocks_k;
  g.chain = chain_blocks(p);
  g.tiles_i = (ei + 127) / 128;
  g.desc = mma_desc(128, c.bn, p.bf16, oi.mn_major, oj.mn_major);
  g.transposed = c.transposed;
  const uint64_t tiles = (uint64_t)g.tiles_i * ((ej + c.bn - 1) / c.bn);
  if (tiles * c.splits * c.outer > 0x7FFFFFFFull) return cudaErrorInvalidValue;
  g.stages = stages_for(tile_bytes(c.bn, oj.mn_major), tiles * c.splits * c.outer <= (uint64_t)sm_count());
  g.tiles = (uint32_t)tiles;
  g.outer = c.outer;
  const uint32_t ld = (p.ep.cols + 7) / 8 * 8;
  if (c.outer > 1) {
    g.partial_step = (uint64_t)p.ep.rows * ld;
    Epilogue& e = g.ep;
    e.out = p.partial, e.ld_out = ld, e.out_dtype = GD_DTYPE_FP32;
    e.bias = e.add = nullptr, e.pre = nullptr;
    e.activation = GD_ACT_NONE;
    e.vectors = 1;
    g.chain = kChainBlocks;                          // (partial sums are fp32 results)
  }
  const uint32_t groups = (uint32_t)tiles * c.outer;
  cudaError_t e;
  if (oi.mn_major) e = oj.mn_major ? launch_bn<true, true>(c.bn, c.splits, g, groups, stream) : launch_bn<true, false>(c.bn, c.splits, g, groups, stream);
  else e = oj.mn_major ? launch_bn<false, true>(c.bn, c.splits, g, groups, stream) : launch_bn<false, false>(c.bn, c.splits, g, groups, stream);
  if (e != cudaSuccess || c.outer == 1) return e;
  note_launches(1);
  return launch_dependent(join_kernel, dim3((uint32_t)((g.partial_step / 8 + 255) / 256)), dim3(256), 0, stream, p.ep, (const float*)p.partial, g.partial_step, ld, c.outer);
}

}  // namespace gd
