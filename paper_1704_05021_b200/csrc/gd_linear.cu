// The linear layer (gd_linear_forward, gd_linear_backward): argument checks, the layout of ragged operands, the activation's
// slope with the bias gradient, and the products (gd_product_split.cu, gd_product_pair.cu).
#include <algorithm>
#include <cmath>
#include <cstring>

#include "gd_linear.cuh"

namespace gd {

SplitChoice choose_product_split(const Product& p);
cudaError_t launch_product_split(const Product& p, const SplitChoice& c, cudaStream_t stream);
cudaError_t launch_product_pair(const Product& p, uint32_t bn, cudaStream_t stream);

namespace {
// Estimated cycles of the pairs' kernel with tiles of 256 x bn: 600 (440) per k block of which the products take 512 (256), not less than an
// epilogue takes, times the waves, and the first copies, the last epilogue and the launch.  Narrow tiles pay where wide ones leave
// pairs without work: weights of 1500 x 1000 over 4000 rows 28.9 against 35.2 us (split kernel 33.4); 8192 x 4096 x 4096 262 against 175.
double cost_product_pair(const Product& p, uint32_t bn) {
  const double tiles = std::ceil(p.ep.rows / 256.0) * std::ceil(p.ep.cols / (double)bn), blocks_k = std::ceil(p.depth / (double)kBlockK);
  const double full = tiles / (sm_count() / 2), waves = p.followed ? std::max(1.0, full) : std::ceil(full);
  return bn == 256 ? 12600.0 + waves * std::max(600.0 * blocks_k, 9000.0) : 10500.0 + waves * std::max(440.0 * blocks_k, 6000.0);
}
}  // namespace

// Tiled-copy map of an operand.  The encoder is the driver's; it is asked for through the runtime, so that the library does not link
// against libcuda and loads on a machine without a GPU.
static bool encode(CUtensorMap* map, const void* p, uint64_t row_bytes, uint64_t width, uint64_t height, uint32_t box_width, uint32_t box_height, int dtype,
                   CUtensorMapSwizzle swizzle) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                              const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static std::atomic<void*> found{nullptr};
  void* f = found.load(std::memory_order_acquire);
  if (!f) {
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) != cudaSuccess || q != cudaDriverEntryPointSuccess || !f)
      return false;
    found.store(f, std::memory_order_release);
  }
  const cuuint64_t dims[2] = {width, height}, strides[1] = {row_bytes};
  const cuuint32_t box[2] = {box_width, box_height}, steps[2] = {1, 1};
  const CUtensorMapDataType type = dtype == GD_DTYPE_FP32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32
                                   : dtype == GD_DTYPE_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                                            : CU_TENSOR_MAP_DATA_TYPE_FLOAT16;
  return reinterpret_cast<Encode>(f)(map, type, 2, const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle,
                                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
static bool encode_tile(CUtensorMap* map, const void* p, uint64_t row_bytes, uint64_t width, uint64_t height, uint32_t box_width, uint32_t box_height, int dtype) {
  return encode(map, p, row_bytes, width, height, box_width, box_height, dtype, CU_TENSOR_MAP_SWIZZLE_128B);
}
bool encode_matrix(CUtensorMap* map, const void* p, uint64_t row_bytes, uint64_t width, uint64_t height, uint32_t box_width, uint32_t box_height, int dtype) {
  return encode(map, p, row_bytes, width, height, box_width, box_height, dtype, CU_TENSOR_MAP_SWIZZLE_NONE);
}
bool encode_operand(CUtensorMap* map, const Operand& o, uint32_t extent, uint32_t depth, uint32_t box_extent, bool bf16) {
  return encode_tile(map, o.p, o.ld * 2, o.mn_major ? extent : depth, o.mn_major ? depth : extent, 64, box_extent, bf16 ? GD_DTYPE_BF16 : GD_DTYPE_FP16);
}
bool encode_piece(CUtensorMap* map, const void* p, uint64_t ld, const Epilogue& ep, uint32_t cols, int dtype) {
  const uint64_t item = dtype == GD_DTYPE_FP32 ? 4 : 2;
  return encode_tile(map, p, (ep.rows > 1 ? ld : (ep.cols + 7) / 8 * 8) * item, cols, ep.rows, (uint32_t)(128 / item), 32, dtype);
}

cudaError_t launch_product(const Product& p, cudaStream_t stream) {
  if (p.ep.rows == 0 || p.ep.cols == 0) return cudaSuccess;
  const SplitChoice split = choose_product_split(p);
  const double wide = cost_product_pair(p, 256), narrow = cost_product_pair(p, 128);
  const bool pair = p.depth && std::min(wide, narrow) < split.cost;
  ProfileScope ps(stream, !pair ? PT_LINEAR : wide <= narrow ? PT_LINEAR_PAIR : PT_LINEAR_PAIR_NARROW);
  const cudaError_t e = pair ? launch_product_pair(p, wide <= narrow ? 256 : 128, stream) : launch_product_split(p, split, stream);
  if (e == cudaSuccess) note_launches(1);
  return e;
}

namespace {

constexpr uint32_t kPackThreads = 256;
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const __grid_constant__ Packs all) {
  pdl_wait();
  pdl_trigger();
  pack_rows(all, (uint64_t)blockIdx.x * kPackThreads + threadIdx.x, (uint64_t)gridDim.x * kPackThreads);
}

// ---------------------------------------------------------------- dz and db
// dz = dy * act'(pre), rounded to the operands' type, and the sums of its columns before that rounding, in one pass over dy and pre;
// ragged operands of the products that follow are laid out by the same launch, in CTAs of their own.
// A cluster of 1 .. 8 CTAs takes `width` columns (64, or 32 where 64 would leave SMs without a CTA), each CTA a share of the rows; a
// thread takes 8 neighbouring columns of every so many rows.  The threads' sums meet by shuffles and in shared memory, the CTAs' are sent
// to the first of the cluster and counted there, always in the same order: no atomics, no second launch.  Bound by the bytes (dy and
// pre read, dz written) where there are many columns, by the 25 instructions an entry of GELU or SiLU takes where there are few.
constexpr uint32_t kSlopeCtas = 8, kSlopeThreads = 512, kSlopeWarps = kSlopeThreads / 32;
struct SlopeArgs {
  const void* dy;
  const void* pre;
  void* dz;            // NULL: only the sums are wanted
  float* db;           // NULL: only dz is wanted
  uint64_t ld_dy, ld_pre, ld_dz;
  uint32_t rows, cols, width, split, ctas;      // split: CTAs of a cluster; ctas: those that take columns; the others lay out `packs`
  int32_t activation;
  uint32_t accumulate, vectors;
  int* status;
  uint64_t budget_ns;  // of the wait for the other CTAs' sums
  uint32_t missing;    // bytes awaited that nobody sends (0; the self-test's 8)
  Packs packs;
};
// Eight 16-bit elements from column c of a row that starts anywhere: the two aligned vectors around them, moved into place. Both lie within
// the row where `inner` holds; a row's ends are read element by element.
__device__ __forceinline__ bool inner(uint32_t c, uint32_t cols) { return c >= 8 && c + 16 <= cols; }
struct Around {
  uint4 lo, hi;
};
__device__ __forceinline__ Around load_around(const uint16_t* s) {
  const uint4* at = reinterpret_cast<const uint4*>((uintptr_t)s & ~(uintptr_t)15);
  return Around{at[0], at[1]};
}
__device__ __forceinline__ uint4 into_place(const Around& a, const uint16_t* s) {
  const uint32_t off = (uint32_t)(uintptr_t)s & 15u;
  uint32_t w[8] = {a.lo.x, a.lo.y, a.lo.z, a.lo.w, a.hi.x, a.hi.y, a.hi.z, a.hi.w};
#pragma unroll
  for (int j = 0; j < 6; ++j) w[j] = off & 8u ? w[j + 2] : w[j];
#pragma unroll
  for (int j = 0; j < 5; ++j) w[j] = off & 4u ? w[j + 1] : w[j];
  const uint32_t bits = (off & 2u) * 8u;
  return make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits));
}
// RAGGED: rows of kWideRow columns and more that start anywhere, read by `load_around`; shorter ones are read element by element, two rows at a
// time.  Backward of 6563 x 1120 <- 3347 155 against 197 us, column sums of 2000 x 85001 138 against 182; slopes of 6214 x 38 14.6
// against 12.6, of 11506 x 433 26.9 against 25.2 (few loads in hand and many ends).
constexpr uint32_t kWideRow = 1024;
template <int DT, bool RAGGED>
__global__ void __launch_bounds__(kSlopeThreads, 2) slope_kernel(const __grid_constant__ SlopeArgs a) {
  constexpr uint32_t kAhead = RAGGED ? 1 : 2;         // rows in hand (two ragged ones do not fit the registers)
  __shared__ float s_sum[kSlopeWarps][64];
  __shared__ __align__(8) float s_all[kSlopeCtas][64];
  __shared__ uint64_t s_in;
  __shared__ int s_never;
  // (a launch without clusters - split = 1 - executes none of their instructions)
  const bool clustered = a.split > 1;
  const uint32_t rank = clustered ? cluster_rank() : 0u, tid = threadIdx.x, lane = tid & 31u, groups = a.width / 8u;      // groups: threads side by side in a row
  const bool pack = blockIdx.x >= a.ctas;
  if (clustered) {
    if (tid == 0) {
      s_never = 0;
      mbar_init(&s_in, 1u);
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
      if (rank == 0) mbar_arrive_expect_tx(&s_in, a.split * a.width * 4u + a.missing);
    }
    __syncthreads();
    cluster_arrive_relaxed();
  }
  pdl_wait();
  pdl_trigger();
  if (pack) {
    pack_rows(a.packs, (uint64_t)(blockIdx.x - a.ctas) * kSlopeThreads + tid, (uint64_t)(gridDim.x - a.ctas) * kSlopeThreads);
    if (clustered) {
      cluster_wait();
      cluster_arrive_relaxed();
      cluster_wait();
    }
    return;
  }
  const uint32_t col0 = blockIdx.x / a.split * a.width, c = col0 + tid % groups * 8u, step = kSlopeThreads / groups;
  const uint32_t per = (a.rows + a.split - 1) / a.split, r0 = min(rank * per, a.rows), r1 = min(r0 + per, a.rows);
  const bool whole = RAGGED ? inner(c, a.cols) : a.vectors && c + 8 <= a.cols;
  const uint16_t *dy = static_cast<const uint16_t*>(a.dy) + c, *pre = static_cast<const uint16_t*>(a.pre) + c;
  float sum[8] = {};
  if (c < a.cols) {
    for (uint32_t first = r0 + tid / groups; first < r1; first += kAhead * step) {
      uint4 gq[kAhead], zq[kAhead];
      Around ga[kAhead], za[kAhead];
      float g[8], z[8];
      if (whole) {
#pragma unroll
        for (uint32_t u = 0; u < kAhead; ++u) {      // these rows' loads are under way together
          const uint64_t r = first + u * step;
          if (r >= r1) break;
          if constexpr (RAGGED) {
            ga[u] = load_around(dy + r * a.ld_dy);
            if (a.activation != GD_ACT_NONE) za[u] = load_around(pre + r * a.ld_pre);
          } else {
            gq[u] = __ldcs(reinterpret_cast<const uint4*>(dy + r * a.ld_dy));
            if (a.activation != GD_ACT_NONE) zq[u] = __ldcs(reinterpret_cast<const uint4*>(pre + r * a.ld_pre));
          }
        }
      }
#pragma unroll
      for (uint32_t u = 0; u < kAhead; ++u) {
        const uint64_t r = first + u * step;
        if (r >= r1) break;
        if (whole) {
          if constexpr (RAGGED) {
            gq[u] = into_place(ga[u], dy + r * a.ld_dy);
            if (a.activation != GD_ACT_NONE) zq[u] = into_place(za[u], pre + r * a.ld_pre);
          }
          widen8(gq[u], DT, g);
          if (a.activation != GD_ACT_NONE) widen8(zq[u], DT, z);
        } else {
#pragma unroll
          for (uint32_t j = 0; j < 8; ++j) {
            const bool in = c + j < a.cols;
            g[j] = in ? load_as(a.dy, r * a.ld_dy + c + j, DT) : 0.f;
            z[j] = in && a.activation != GD_ACT_NONE ? load_as(a.pre, r * a.ld_pre + c + j, DT) : 0.f;
          }
        }
        if (a.activation == GD_ACT_RELU) {
#pragma unroll
          for (int j = 0; j < 8; ++j) g[j] = z[j] > 0.f ? g[j] : 0.f * g[j];
        } else if (a.activation == GD_ACT_GELU) {
#pragma unroll
          for (int j = 0; j < 8; ++j) g[j] *= gelu_slope(z[j]);
        } else if (a.activation == GD_ACT_SILU) {
#pragma unroll
          for (int j = 0; j < 8; ++j) g[j] *= silu_slope(z[j]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += g[j];
        // (dz's own rows are padded to a multiple of 8 with zeros, which the ragged case above made)
        if (a.dz) store8_as(a.dz, r * a.ld_dz + c, DT, g);
      }
    }
  }
  if (a.db) {
    for (uint32_t o = groups; o < 32u; o *= 2) {
#pragma unroll
      for (int j = 0; j < 8; ++j) sum[j] += __shfl_xor_sync(0xFFFFFFFFu, sum[j], o);
    }
    if (lane < groups) {
#pragma unroll
      for (int j = 0; j < 8; ++j) s_sum[tid >> 5][lane * 8u + j] = sum[j];
    }
    __syncthreads();
    if (!clustered) {
      if (tid < a.width) {
        float t = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < kSlopeWarps; ++w) t += s_sum[w][tid];
        const uint32_t col = col0 + tid;
        if (col < a.cols) a.db[col] = a.accumulate ? a.db[col] + t : t;
      }
      return;
    }
    cluster_wait();                                  // (the first CTA's mbarrier exists)
    if (tid < a.width / 2) {
      float2 t = make_float2(0.f, 0.f);
#pragma unroll
      for (uint32_t w = 0; w < kSlopeWarps; ++w) t.x += s_sum[w][2 * tid], t.y += s_sum[w][2 * tid + 1];
      send_peer2(peer_address(smem_u32(&s_all[rank][2 * tid]), 0), t, peer_address(smem_u32(&s_in), 0));
    }
    if (rank == 0 && tid < a.width) {
      const bool there = mbar_wait(&s_in, 0u, &s_never, a.budget_ns);
      if (!there) atomicExch(a.status, GD_ERR_DEVICE_TIMEOUT);
      float t = there ? 0.f : NAN;
      for (uint32_t q = 0; q < a.split; ++q) t += s_all[q][tid];
      const uint32_t col = col0 + tid;
      if (col < a.cols) a.db[col] = a.accumulate ? a.db[col] + t : t;
    }
  } else if (clustered) {
    cluster_wait();
  }
  if (clustered) {
    cluster_arrive_relaxed();                        // (nobody leaves while something may still be on its way to it)
    cluster_wait();
  }
}
cudaError_t launch_slope(SlopeArgs& a, int dtype, cudaStream_t stream) {
  ProfileScope ps(stream, PT_LINEAR_SLOPE);
  // CTAs for every SM twice over, if there are rows enough for a CTA's threads
  a.width = (a.cols + 63) / 64 * kSlopeCtas < 2u * sm_count() ? 32 : 64;
  const uint32_t tiles = (a.cols + a.width - 1) / a.width;
  a.split = 1;
  while (a.split < kSlopeCtas && tiles * a.split < 2u * sm_count() && a.rows > a.split * (kSlopeThreads * 8u / a.width)) a.split *= 2;
  a.ctas = tiles * a.split;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(a.ctas + (pack_ctas(a.packs, kSlopeThreads) + a.split - 1) / a.split * a.split);
  cfg.blockDim = dim3(kSlopeThreads);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = a.split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = a.split > 1 ? 2 : 1;
  const bool bf16 = dtype == GD_DTYPE_BF16, ragged = !a.vectors && a.cols >= kWideRow;
  const cudaError_t e = !ragged ? cudaLaunchKernelEx(&cfg, bf16 ? slope_kernel<GD_DTYPE_BF16, false> : slope_kernel<GD_DTYPE_FP16, false>, a)
                                : cudaLaunchKernelEx(&cfg, bf16 ? slope_kernel<GD_DTYPE_BF16, true> : slope_kernel<GD_DTYPE_FP16, true>, a);
  if (e == cudaSuccess) note_launches(1);
  return e;
}

// ---------------------------------------------------------------- host side
int check_shape(uint64_t m, uint64_t n, uint64_t k, int dtype, int act, int layout) {
  if (!is_16bit(dtype) || act < GD_ACT_NONE || act > GD_ACT_SILU || (layout != GD_W_IN_OUT && layout != GD_W_OUT_IN)) return GD_ERR_INVALID_ARG;
  if (m >> 31 || n >> 31 || k >> 31) return GD_ERR_TOO_LARGE;
  return GD_OK;
}

int forward(const gd_linear_forward_args* a, cudaStream_t stream) {
  if (!a || a->reserved != 0) return GD_ERR_INVALID_ARG;
  int rc = check_shape(a->m, a->n, a->k, a->dtype, a->activation, a->w_layout);
  if (rc != GD_OK) return rc;
  if ((a->y_dtype != a->dtype && a->y_dtype != GD_DTYPE_FP32) || (a->bias && a->bias_dtype != a->dtype && a->bias_dtype != GD_DTYPE_FP32)) return GD_ERR_INVALID_ARG;
  if (a->m == 0 || a->n == 0) return GD_OK;
  const bool in_out = a->w_layout == GD_W_IN_OUT;
  const uint64_t w_rows = in_out ? a->k : a->n, w_cols = in_out ? a->n : a->k;
  if (a->k && (!good_rows(a->x, a->ldx, a->m, a->k, 2) || !good_rows(a->w, a->ldw, w_rows, w_cols, 2))) return GD_ERR_INVALID_ARG;
  if (!good_rows(a->y, a->ldy, a->m, a->n, dtype_bytes(a->y_dtype)) || (a->bias && !aligned_to(a->bias, dtype_bytes(a->bias_dtype))) ||
      (a->residual && !good_rows(a->residual, a->ld_residual, a->m, a->n, 2)) || (a->pre && !good_rows(a->pre, a->ld_pre, a->m, a->n, 2)))
    return GD_ERR_INVALID_ARG;
  if (a->residual == a->y && (a->y_dtype != a->dtype || (a->m > 1 && a->ldy != a->ld_residual))) return GD_ERR_INVALID_ARG;
  if (check_workspace(a->workspace, a->workspace_bytes) != GD_OK) return GD_ERR_WORKSPACE;
  Workspace ws{(unsigned char*)a->workspace, kStatusBytes, a->workspace_bytes};
  Packs packs;
  packs.count = 0;
  Product p;
  std::memset(&p, 0, sizeof(p));
  if ((rc = partial_place(a->k, ws, &p.partial)) != GD_OK) return rc;
  if ((rc = operand(a->x, a->ldx, a->m, a->k, ws, &packs, &p.a)) != GD_OK || (rc = operand(a->w, a->ldw, w_rows, w_cols, ws, &packs, &p.b)) != GD_OK) return rc;
  p.b.mn_major = in_out;
  p.depth = (uint32_t)a->k;
  p.bf16 = a->dtype == GD_DTYPE_BF16;
  p.status = (int*)a->workspace;
  Epilogue& e = p.ep;
  e.out = a->y, e.ld_out = a->ldy, e.out_dtype = a->y_dtype;
  e.bias = a->bias, e.bias_dtype = a->bias_dtype;
  e.add = a->residual, e.ld_add = a->ld_residual, e.add_dtype = a->dtype;
  e.pre = a->pre, e.ld_pre = a->ld_pre, e.dtype = a->dtype;
  e.rows = (uint32_t)a->m, e.cols = (uint32_t)a->n;
  e.activation = a->activation;
  const bool one = a->m == 1;
  e.vectors = vector_rows(e.out, one ? 8 : e.ld_out, e.out_dtype) && vector_rows(e.bias, 8, GD_DTYPE_FP32) && vector_rows(e.add, one ? 8 : e.ld_add, e.add_dtype) &&
              vector_rows(e.pre, one ? 8 : e.ld_pre, e.dtype);
  e.pairs = paired_rows(e.out, one ? 8 : e.ld_out, e.out_dtype) && paired_rows(e.add, one ? 8 : e.ld_add, e.add_dtype) && paired_rows(e.pre, one ? 8 : e.ld_pre, e.dtype);
  return launch_pack(packs, stream) == cudaSuccess && launch_product(p, stream) == cudaSuccess ? GD_OK : GD_ERR_CUDA;
}

int backward(const gd_linear_backward_args* a, cudaStream_t stream) {
  if (!a || a->reserved != 0 || (a->flags & ~(uint32_t)GD_LINEAR_ACCUMULATE)) return GD_ERR_INVALID_ARG;
  int rc = check_shape(a->m, a->n, a->k, a->dtype, a->activation, a->w_layout);
  if (rc != GD_OK) return rc;
  const bool in_out = a->w_layout == GD_W_IN_OUT, add = (a->flags & GD_LINEAR_ACCUMULATE) != 0, slope = a->activation != GD_ACT_NONE;
  const uint64_t m = a->m, n = a->n, k = a->k, w_rows = in_out ? k : n, w_cols = in_out ? n : k;
  if ((a->dw_dtype != a->dtype && a->dw_dtype != GD_DTYPE_FP32) || (a->dw && add && a->dw_dtype != GD_DTYPE_FP32)) return GD_ERR_INVALID_ARG;
  const bool has_dx = a->dx && m && k, has_dw = a->dw && n && k, has_db = a->db && n;
  if (!has_dx && !has_dw && !has_db) return GD_OK;
  if (m && n && (!good_rows(a->dy, a->ld_dy, m, n, 2) || (slope && !good_rows(a->pre, a->ld_pre, m, n, 2)))) return GD_ERR_INVALID_ARG;
  if (has_dx && ((n && !good_rows(a->w, a->ldw, w_rows, w_cols, 2)) || !good_rows(a->dx, a->ld_dx, m, k, 2))) return GD_ERR_INVALID_ARG;
  if (has_dw && ((m && !good_rows(a->x, a->ldx, m, k, 2)) || !good_rows(a->dw, a->ld_dw, w_rows, w_cols, dtype_bytes(a->dw_dtype)))) return GD_ERR_INVALID_ARG;
  if (has_db && !aligned_to(a->db, 4)) return GD_ERR_INVALID_ARG;
  if (check_workspace(a->workspace, a->workspace_bytes) != GD_OK) return GD_ERR_WORKSPACE;
  Workspace ws{(unsigned char*)a->workspace, kStatusBytes, a->workspace_bytes};

  // dz: dy itself without an activation (laid out anew if its rows are ragged), else made here together with db
  Operand dz{a->dy, row_step(a->ld_dy, m, n), false};
  const bool products = (has_dx || has_dw) && m && n, make = products && (slope || !tiles_as_it_is(a->dy, dz.ld));
  SlopeArgs s;
  std::memset(&s, 0, sizeof(s));
  if (make) {
    s.dz = ws.take(m, n);
    if (!s.dz) return GD_ERR_WORKSPACE;
    s.ld_dz = up(n, 8);
    dz.p = s.dz, dz.ld = s.ld_dz;
  }
  Operand w{}, x{};
  float* partial = nullptr;
  if ((rc = partial_place(std::max(has_dx ? n : 0, has_dw ? m : 0), ws, &partial)) != GD_OK) return rc;
  s.packs.count = 0;
  if (has_dx && n && (rc = operand(a->w, a->ldw, w_rows, w_cols, ws, &s.packs, &w)) != GD_OK) return rc;
  if (has_dw && m && (rc = operand(a->x, a->ldx, m, k, ws, &s.packs, &x)) != GD_OK) return rc;
  if (make || has_db) {
    s.status = (int*)a->workspace;
    s.budget_ns = kWaitBudgetNs;
    s.dy = a->dy, s.ld_dy = a->ld_dy;
    s.pre = a->pre, s.ld_pre = a->ld_pre;
    s.db = has_db ? a->db : nullptr;
    s.rows = (uint32_t)m, s.cols = (uint32_t)n;
    s.activation = a->activation;
    s.accumulate = add;
    s.vectors = vector_rows(a->dy, row_step(a->ld_dy, m, n), a->dtype) && (!slope || vector_rows(a->pre, row_step(a->ld_pre, m, n), a->dtype));
    if (launch_slope(s, a->dtype, stream) != cudaSuccess) return GD_ERR_CUDA;
  } else if (launch_pack(s.packs, stream) != cudaSuccess) {
    return GD_ERR_CUDA;
  }
  BackProducts q;
  q.dz = dz, q.w = w, q.x = x;
  q.partial = partial;
  q.m = m, q.n = n, q.k = k;
  q.in_out = in_out, q.add = add;
  q.dtype = a->dtype, q.dw_dtype = a->dw_dtype;
  q.dx = has_dx ? a->dx : nullptr, q.ld_dx = a->ld_dx;
  q.dw = has_dw ? a->dw : nullptr, q.ld_dw = a->ld_dw;
  q.status = (int*)a->workspace;
  return launch_back_products(q, stream) == cudaSuccess ? GD_OK : GD_ERR_CUDA;
}

}  // namespace

cudaError_t launch_pack(const Packs& all, cudaStream_t stream) {
  if (all.count == 0) return cudaSuccess;
  ProfileScope ps(stream, PT_LINEAR_PACK);
  const cudaError_t e = launch_dependent(pack_kernel, dim3(pack_ctas(all, kPackThreads)), dim3(kPackThreads), 0, stream, all);
  if (e == cudaSuccess) note_launches(1);
  return e;
}

cudaError_t launch_back_products(const BackProducts& q, cudaStream_t stream) {
  const uint64_t m = q.m, n = q.n, k = q.k, w_rows = q.in_out ? k : n, w_cols = q.in_out ? n : k;
  const bool has_dx = q.dx != nullptr, has_dw = q.dw != nullptr;
  Product p;
  std::memset(&p, 0, sizeof(p));
  p.bf16 = q.dtype == GD_DTYPE_BF16;
  p.status = q.status;
  p.ep.dtype = q.dtype;
  if (has_dx) {                       // dx = dz W^T: contraction over n
    p.a = q.dz, p.a.mn_major = false;
    p.b = q.w, p.b.mn_major = !q.in_out;
    p.depth = (uint32_t)n;
    p.partial = n >= kLongDepth ? q.partial : nullptr;
    p.followed = has_dw && n < kLongDepth;
    p.ep.out = q.dx, p.ep.ld_out = q.ld_dx, p.ep.out_dtype = q.dtype;
    p.ep.rows = (uint32_t)m, p.ep.cols = (uint32_t)k;
    p.ep.vectors = vector_rows(q.dx, row_step(q.ld_dx, m, k), q.dtype);
    p.ep.pairs = paired_rows(q.dx, row_step(q.ld_dx, m, k), q.dtype);
    const cudaError_t e = launch_product(p, stream);
    if (e != cudaSuccess) return e;
  }
  if (has_dw) {                       // dw = x^T dz, or its transpose: contraction over m
    p.a = q.in_out ? q.x : q.dz, p.b = q.in_out ? q.dz : q.x;
    p.a.mn_major = p.b.mn_major = true;
    p.depth = (uint32_t)m;
    p.partial = m >= kLongDepth ? q.partial : nullptr;     // (the product before this one has been joined by the time it is written)
    p.ep.out = q.dw, p.ep.ld_out = q.ld_dw, p.ep.out_dtype = q.dw_dtype;
    p.ep.rows = (uint32_t)w_rows, p.ep.cols = (uint32_t)w_cols;
    p.followed = false;
    p.beside = has_dx && n < kLongDepth;                  // (a joined dx has a launch in between, and the partial sums' place)
    if (q.add) p.ep.add = q.dw, p.ep.ld_add = q.ld_dw, p.ep.add_dtype = GD_DTYPE_FP32;
    p.ep.vectors = vector_rows(q.dw, row_step(q.ld_dw, w_rows, w_cols), q.dw_dtype);
    p.ep.pairs = paired_rows(q.dw, row_step(q.ld_dw, w_rows, w_cols), q.dw_dtype);
    const cudaError_t e = launch_product(p, stream);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

}  // namespace gd

extern "C" {

int gd_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, int any_layout, size_t* bytes_out) {
  using namespace gd;
  if (!bytes_out) return GD_ERR_INVALID_ARG;
  if (m >> 31 || n >> 31 || k >> 31) return GD_ERR_TOO_LARGE;
  auto matrix = [](uint64_t rows, uint64_t cols) { return up(rows * up(cols, 8) * 2, 256); };
  uint64_t b = kStatusBytes + matrix(m, n);                              // dz
  if (std::max(m, std::max(n, k)) >= kLongDepth) b += kPartialBytes;      // partial sums of a long contraction
  if (any_layout || k % 8) b += matrix(m, k);                            // x
  if (any_layout || k % 8 || n % 8) b += std::max(matrix(k, n), matrix(n, k));   // w, in either layout
  *bytes_out = (size_t)b;
  return GD_OK;
}

int gd_linear_status(const void* workspace, void* stream) {
  if (!workspace) return GD_ERR_INVALID_ARG;
  int status = 0;
  if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return GD_ERR_CUDA;
  if (cudaMemcpy(&status, workspace, sizeof(int), cudaMemcpyDeviceToHost) != cudaSuccess) return GD_ERR_CUDA;
  return status;
}

int gd_selftest_linear_wait(void* workspace, size_t workspace_bytes, uint64_t budget_ns, void* stream) {
  using namespace gd;
  constexpr uint32_t rows = 256, cols = 32;              // two CTAs in a cluster
  constexpr size_t sums = kStatusBytes, values = sums + 256;
  if (check_workspace(workspace, workspace_bytes) != GD_OK || workspace_bytes < values + rows * cols * 2) return GD_ERR_WORKSPACE;
  unsigned char* base = (unsigned char*)workspace;
  if (cudaMemsetAsync(base, 0, values + rows * cols * 2, (cudaStream_t)stream) != cudaSuccess) return GD_ERR_CUDA;
  SlopeArgs s;
  std::memset(&s, 0, sizeof(s));
  s.dy = base + values, s.ld_dy = cols;
  s.db = (float*)(base + sums);
  s.rows = rows, s.cols = cols;
  s.activation = GD_ACT_NONE;
  s.vectors = 1;
  s.status = (int*)workspace;
  s.budget_ns = budget_ns;
  s.missing = 8;
  return launch_slope(s, GD_DTYPE_BF16, (cudaStream_t)stream) == cudaSuccess ? GD_OK : GD_ERR_CUDA;
}

int gd_linear_forward(const gd_linear_forward_args* a, void* stream) { return gd::forward(a, (cudaStream_t)stream); }

int gd_linear_backward(const gd_linear_backward_args* a, void* stream) { return gd::backward(a, (cudaStream_t)stream); }

}  // extern "C"
