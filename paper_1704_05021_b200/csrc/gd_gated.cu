// The gated feed-forward block (gd_gated_forward, gd_gated_backward): argument checks, ragged operands, the way back through activation and
// product with the bias gradient; the products are in gd_gated_product.cu (forward) and those of the linear layer (backward).
#include <algorithm>
#include <cstring>

#include "gd_gated.cuh"
#include "gd_layers.h"

namespace gd {
namespace {

// ---------------------------------------------------------------- dz and db
// dz = [dy * u * act'(a), dy * act(a)], rounded to the operands' type, and the sums of its columns before that rounding, in one pass over dy and
// pre = [a, u]; ragged operands of the products that follow are laid out by the same launch, in CTAs of their own.  As in the linear layer: a
// cluster of 1 .. 8 CTAs takes `width` columns of dy, each CTA a share of the rows, a thread 8 neighbouring columns of every so many rows; the
// sums meet by shuffles, in shared memory and, sent and counted, in the cluster's first CTA, always in the same order.
// Bound by the bytes: three values read and two written for each of dy.
constexpr uint32_t kSlopeCtas = 8, kSlopeThreads = 256, kSlopeWarps = kSlopeThreads / 32;
struct SlopeArgs {
  const void* dy;
  const void* pre;
  void* dz;            // NULL: only the sums are wanted
  float* db;           // NULL: only dz is wanted
  uint64_t ld_dy, ld_pre, ld_dz;
  uint32_t rows, cols, width, split, ctas;      // cols: of dy; split: CTAs of a cluster; ctas: those that take columns; the others lay out `packs`
  int32_t activation;
  uint32_t accumulate, vectors;
  int* status;
  uint64_t budget_ns;  // of the wait for the other CTAs' sums
  uint32_t missing;    // bytes awaited that nobody sends (0; the self-test's 8)
  Packs packs;
};
// (a, u, g) -> the two halves of dz, in a's and u's place
__device__ __forceinline__ void back8(float (&a)[8], float (&u)[8], const float (&g)[8], int act) {
  float v[8];
  if (act == GD_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = a[j] < 0.f ? 0.f : a[j], a[j] = a[j] > 0.f ? 1.f : 0.f;
  } else if (act == GD_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = gelu_both(a[j], &v[j]);
  } else if (act == GD_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = silu_both(a[j], &v[j]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = a[j], a[j] = 1.f;
  }
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    a[j] *= g[j] * u[j];
    u[j] = g[j] * v[j];
  }
}
template <int DT>
__global__ void __launch_bounds__(kSlopeThreads, 3) gated_slope_kernel(const __grid_constant__ SlopeArgs a) {
  __shared__ float s_sum[kSlopeWarps][2][64];
  __shared__ __align__(8) float s_all[kSlopeCtas][128];
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
      if (rank == 0) mbar_arrive_expect_tx(&s_in, a.split * a.width * 8u + a.missing);
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
  const uint16_t *dy = static_cast<const uint16_t*>(a.dy) + c, *pre = static_cast<const uint16_t*>(a.pre) + c;
  uint16_t* dz = a.dz ? static_cast<uint16_t*>(a.dz) + c : nullptr;
  float sum[2][8] = {};
  if (c < a.cols) {
    if (a.vectors) {
      constexpr uint32_t kInHand = 2;                  // rows
      uint4 gq[kInHand], aq[kInHand], uq[kInHand];
      const auto ask = [&](uint64_t r, uint32_t q) {
        if (r >= r1) return;
        gq[q] = __ldcs(reinterpret_cast<const uint4*>(dy + r * a.ld_dy));
        aq[q] = __ldcs(reinterpret_cast<const uint4*>(pre + r * a.ld_pre));
        uq[q] = __ldcs(reinterpret_cast<const uint4*>(pre + r * a.ld_pre + a.cols));
      };
      const uint64_t from = r0 + tid / groups;
#pragma unroll
      for (uint32_t q = 0; q < kInHand; ++q) ask(from + q * step, q);
      for (uint64_t first = from; first < r1; first += kInHand * step) {
#pragma unroll
        for (uint32_t q = 0; q < kInHand; ++q) {
          const uint64_t r = first + q * step;
          if (r >= r1) break;
          float g[8], z[8], u[8];
          widen8_t<DT>(gq[q], g), widen8_t<DT>(aq[q], z), widen8_t<DT>(uq[q], u);
          ask(r + kInHand * step, q);
          back8(z, u, g, a.activation);
#pragma unroll
          for (int j = 0; j < 8; ++j) sum[0][j] += z[j], sum[1][j] += u[j];
          if (dz) {
            *reinterpret_cast<uint4*>(dz + r * a.ld_dz) = narrow8_t<DT>(z);
            *reinterpret_cast<uint4*>(dz + r * a.ld_dz + a.cols) = narrow8_t<DT>(u);
          }
        }
      }
    } else {
      const uint32_t live = min(a.cols - c, 8u);
      for (uint64_t r = r0 + tid / groups; r < r1; r += step) {
        float g[8], z[8], u[8];
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          const bool in = j < live;
          g[j] = in ? load_as(dy, r * a.ld_dy + j, DT) : 0.f;
          z[j] = in ? load_as(pre, r * a.ld_pre + j, DT) : 0.f;
          u[j] = in ? load_as(pre, r * a.ld_pre + a.cols + j, DT) : 0.f;
        }
        back8(z, u, g, a.activation);
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          if (j >= live) continue;
          sum[0][j] += z[j], sum[1][j] += u[j];
          if (dz) store_as(dz, r * a.ld_dz + j, DT, z[j]), store_as(dz, r * a.ld_dz + a.cols + j, DT, u[j]);
        }
      }
    }
  }
  if (a.db) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      for (uint32_t o = groups; o < 32u; o *= 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[h][j] += __shfl_xor_sync(0xFFFFFFFFu, sum[h][j], o);
      }
      if (lane < groups) {
#pragma unroll
        for (int j = 0; j < 8; ++j) s_sum[tid >> 5][h][lane * 8u + j] = sum[h][j];
      }
    }
    __syncthreads();
    // sums 0 .. width - 1 are the gate's columns, the next `width` the others'
    const uint32_t h = tid / a.width, i = tid % a.width, col = col0 + i;
    if (!clustered) {
      if (h < 2 && col < a.cols) {
        float t = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < kSlopeWarps; ++w) t += s_sum[w][h][i];
        float* to = a.db + (uint64_t)h * a.cols + col;
        *to = a.accumulate ? *to + t : t;
      }
      return;
    }
    cluster_wait();                                  // (the first CTA's mbarrier exists)
    if (tid < a.width) {
      const uint32_t p = 2 * tid, ph = p / a.width, pi = p % a.width;
      float2 t = make_float2(0.f, 0.f);
#pragma unroll
      for (uint32_t w = 0; w < kSlopeWarps; ++w) t.x += s_sum[w][ph][pi], t.y += s_sum[w][ph][pi + 1];
      send_peer2(peer_address(smem_u32(&s_all[rank][p]), 0), t, peer_address(smem_u32(&s_in), 0));
    }
    if (rank == 0 && h < 2) {
      const bool there = mbar_wait(&s_in, 0u, &s_never, a.budget_ns);
      if (!there) atomicExch(a.status, GD_ERR_DEVICE_TIMEOUT);
      float t = there ? 0.f : NAN;
      for (uint32_t q = 0; q < a.split; ++q) t += s_all[q][tid];
      float* to = a.db + (uint64_t)h * a.cols + col;
      if (col < a.cols) *to = a.accumulate ? *to + t : t;
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
  ProfileScope ps(stream, PT_GATED_SLOPE);
  // CTAs for every SM, if there are rows enough for a CTA's threads (4000 x 2048: 20 us by 64 columns, 24 by twice as many CTAs of 32)
  a.width = (a.cols + 63) / 64 * kSlopeCtas < (uint32_t)sm_count() ? 32 : 64;
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
  const cudaError_t e = cudaLaunchKernelEx(&cfg, dtype == GD_DTYPE_BF16 ? gated_slope_kernel<GD_DTYPE_BF16> : gated_slope_kernel<GD_DTYPE_FP16>, a);
  if (e == cudaSuccess) note_launches(1);
  return e;
}

// ---------------------------------------------------------------- host side
int check_shape(uint64_t m, uint64_t n, uint64_t k, int dtype, int act, int layout) {
  if (!is_16bit(dtype) || act < GD_ACT_NONE || act > GD_ACT_SILU || (layout != GD_W_IN_OUT && layout != GD_W_OUT_IN)) return GD_ERR_INVALID_ARG;
  return m >> 30 || n >> 30 || k >> 30 ? GD_ERR_TOO_LARGE : GD_OK;
}

int forward(const gd_gated_forward_args* a, cudaStream_t stream) {
  if (!a) return GD_ERR_INVALID_ARG;
  int rc = check_shape(a->m, a->n, a->k, a->dtype, a->activation, a->w_layout);
  if (rc != GD_OK) return rc;
  if (a->bias && a->bias_dtype != a->dtype && a->bias_dtype != GD_DTYPE_FP32) return GD_ERR_INVALID_ARG;
  if (a->m == 0 || a->n == 0) return GD_OK;
  const bool in_out = a->w_layout == GD_W_IN_OUT;
  const uint64_t m = a->m, n = a->n, k = a->k;
  if (k && (!good_rows(a->x, a->ldx, m, k, 2) || !good_rows(a->w, a->ldw, in_out ? k : 2 * n, in_out ? 2 * n : k, 2))) return GD_ERR_INVALID_ARG;
  if (!good_rows(a->y, a->ldy, m, n, 2) || (a->pre && !good_rows(a->pre, a->ld_pre, m, 2 * n, 2)) || (a->bias && !aligned_to(a->bias, dtype_bytes(a->bias_dtype))))
    return GD_ERR_INVALID_ARG;
  if (check_workspace(a->workspace, a->workspace_bytes) != GD_OK) return GD_ERR_WORKSPACE;
  Workspace ws{(unsigned char*)a->workspace, kStatusBytes, a->workspace_bytes};
  Packs packs;
  packs.count = 0;
  GatedProduct p;
  std::memset(&p, 0, sizeof(p));
  if ((rc = operand(a->x, a->ldx, m, k, ws, &packs, &p.x)) != GD_OK) return rc;
  // the halves of W: n columns beside each other, or n rows one behind the other; a half that starts at an odd place is laid out anew
  const uint16_t* w = static_cast<const uint16_t*>(a->w);
  const uint64_t ldw = in_out && k <= 1 ? up(2 * n, 8) : a->ldw;
  if (in_out) rc = operand(w, ldw, k, n, ws, &packs, &p.gate) != GD_OK || operand(w + n, ldw, k, n, ws, &packs, &p.up) != GD_OK ? GD_ERR_WORKSPACE : GD_OK;
  else rc = operand(w, ldw, n, k, ws, &packs, &p.gate) != GD_OK || operand(w + n * ldw, ldw, n, k, ws, &packs, &p.up) != GD_OK ? GD_ERR_WORKSPACE : GD_OK;
  if (rc != GD_OK) return rc;
  p.gate.mn_major = p.up.mn_major = in_out;
  p.depth = (uint32_t)k;
  p.bf16 = a->dtype == GD_DTYPE_BF16;
  p.status = (int*)a->workspace;
  GatedEpilogue& e = p.ep;
  e.out = a->y, e.ld_out = row_step(a->ldy, m, n);
  e.pre = a->pre, e.ld_pre = row_step(a->ld_pre, m, 2 * n);
  e.bias = a->bias, e.bias_dtype = a->bias_dtype;
  e.rows = (uint32_t)m, e.cols = (uint32_t)n;
  e.dtype = a->dtype, e.activation = a->activation;
  e.vectors = n % 8 == 0 && vector_rows(e.out, e.ld_out, a->dtype) && vector_rows(e.pre, e.ld_pre, a->dtype);
  return launch_pack(packs, stream) == cudaSuccess && launch_gated_product(p, stream) == cudaSuccess ? GD_OK : GD_ERR_CUDA;
}

int backward(const gd_gated_backward_args* a, cudaStream_t stream) {
  if (!a || a->reserved != 0 || (a->flags & ~(uint32_t)GD_LINEAR_ACCUMULATE)) return GD_ERR_INVALID_ARG;
  int rc = check_shape(a->m, a->n, a->k, a->dtype, a->activation, a->w_layout);
  if (rc != GD_OK) return rc;
  const bool in_out = a->w_layout == GD_W_IN_OUT, add = (a->flags & GD_LINEAR_ACCUMULATE) != 0;
  const uint64_t m = a->m, n = a->n, k = a->k, w_rows = in_out ? k : 2 * n, w_cols = in_out ? 2 * n : k;
  if ((a->dw_dtype != a->dtype && a->dw_dtype != GD_DTYPE_FP32) || (a->dw && add && a->dw_dtype != GD_DTYPE_FP32)) return GD_ERR_INVALID_ARG;
  const bool has_dx = a->dx && m && k, has_dw = a->dw && n && k, has_db = a->db && n;
  if (!has_dx && !has_dw && !has_db) return GD_OK;
  if (m && n && (!good_rows(a->dy, a->ld_dy, m, n, 2) || !good_rows(a->pre, a->ld_pre, m, 2 * n, 2))) return GD_ERR_INVALID_ARG;
  if (has_dx && ((n && !good_rows(a->w, a->ldw, w_rows, w_cols, 2)) || !good_rows(a->dx, a->ld_dx, m, k, 2))) return GD_ERR_INVALID_ARG;
  if (has_dw && ((m && !good_rows(a->x, a->ldx, m, k, 2)) || !good_rows(a->dw, a->ld_dw, w_rows, w_cols, dtype_bytes(a->dw_dtype)))) return GD_ERR_INVALID_ARG;
  if (has_db && !aligned_to(a->db, 4)) return GD_ERR_INVALID_ARG;
  if (check_workspace(a->workspace, a->workspace_bytes) != GD_OK) return GD_ERR_WORKSPACE;
  Workspace ws{(unsigned char*)a->workspace, kStatusBytes, a->workspace_bytes};
  BackProducts q;
  std::memset(&q, 0, sizeof(q));
  SlopeArgs s;
  std::memset(&s, 0, sizeof(s));
  s.packs.count = 0;
  const bool products = (has_dx || has_dw) && m && n;
  if (products) {
    s.dz = ws.take(m, 2 * n);
    if (!s.dz) return GD_ERR_WORKSPACE;
    s.ld_dz = up(2 * n, 8);
    q.dz = Operand{s.dz, s.ld_dz, false};
  }
  if ((rc = partial_place(std::max(has_dx ? 2 * n : 0, has_dw ? m : 0), ws, &q.partial)) != GD_OK) return rc;
  if (has_dx && n && (rc = operand(a->w, a->ldw, w_rows, w_cols, ws, &s.packs, &q.w)) != GD_OK) return rc;
  if (has_dw && m && (rc = operand(a->x, a->ldx, m, k, ws, &s.packs, &q.x)) != GD_OK) return rc;
  if (products || has_db) {
    s.status = (int*)a->workspace;
    s.budget_ns = kWaitBudgetNs;
    s.dy = a->dy, s.ld_dy = row_step(a->ld_dy, m, n);
    s.pre = a->pre, s.ld_pre = row_step(a->ld_pre, m, 2 * n);
    s.db = has_db ? a->db : nullptr;
    s.rows = (uint32_t)m, s.cols = (uint32_t)n;
    s.activation = a->activation;
    s.accumulate = add;
    s.vectors = n % 8 == 0 && vector_rows(a->dy, s.ld_dy, a->dtype) && vector_rows(a->pre, s.ld_pre, a->dtype);
    if (launch_slope(s, a->dtype, stream) != cudaSuccess) return GD_ERR_CUDA;
  } else if (launch_pack(s.packs, stream) != cudaSuccess) {
    return GD_ERR_CUDA;
  }
  q.m = m, q.n = 2 * n, q.k = k;
  q.in_out = in_out, q.add = add;
  q.dtype = a->dtype, q.dw_dtype = a->dw_dtype;
  q.dx = has_dx ? a->dx : nullptr, q.ld_dx = a->ld_dx;
  q.dw = has_dw ? a->dw : nullptr, q.ld_dw = a->ld_dw;
  q.status = (int*)a->workspace;
  return launch_back_products(q, stream) == cudaSuccess ? GD_OK : GD_ERR_CUDA;
}

}  // namespace
}  // namespace gd

extern "C" {

int gd_gated_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, int any_layout, size_t* bytes_out) {
  using namespace gd;
  if (!bytes_out) return GD_ERR_INVALID_ARG;
  if (m >> 30 || n >> 30 || k >> 30) return GD_ERR_TOO_LARGE;
  auto matrix = [](uint64_t rows, uint64_t cols) { return up(rows * up(cols, 8) * 2, 256); };
  uint64_t b = kStatusBytes + matrix(m, 2 * n);                            // dz
  if (std::max(m, std::max(2 * n, k)) >= kLongDepth) b += kPartialBytes;    // partial sums of a long contraction
  if (any_layout || k % 8) b += matrix(m, k);                              // x
  if (any_layout || k % 8 || n % 8)                                        // w whole, or its halves, in either layout
    b += std::max(std::max(matrix(k, 2 * n), matrix(2 * n, k)), std::max(2 * matrix(k, n), 2 * matrix(n, k)));
  *bytes_out = (size_t)b;
  return GD_OK;
}
int gd_gated_forward(const gd_gated_forward_args* a, void* stream) { return gd::forward(a, (cudaStream_t)stream); }
int gd_gated_backward(const gd_gated_backward_args* a, void* stream) { return gd::backward(a, (cudaStream_t)stream); }

int gd_selftest_gated_wait(void* workspace, size_t workspace_bytes, uint64_t budget_ns, void* stream) {
  using namespace gd;
  constexpr uint32_t rows = 128, cols = 32;              // two CTAs in a cluster
  constexpr size_t sums = kStatusBytes, dy = sums + 2 * cols * 4, pre = dy + rows * cols * 2, end = pre + rows * 2 * cols * 2;
  if (check_workspace(workspace, workspace_bytes) != GD_OK || workspace_bytes < end) return GD_ERR_WORKSPACE;
  unsigned char* base = (unsigned char*)workspace;
  if (cudaMemsetAsync(base, 0, end, (cudaStream_t)stream) != cudaSuccess) return GD_ERR_CUDA;
  SlopeArgs s;
  std::memset(&s, 0, sizeof(s));
  s.dy = base + dy, s.ld_dy = cols;
  s.pre = base + pre, s.ld_pre = 2 * cols;
  s.db = (float*)(base + sums);
  s.rows = rows, s.cols = cols;
  s.activation = GD_ACT_SILU;
  s.vectors = 1;
  s.status = (int*)workspace;
  s.budget_ns = budget_ns;
  s.missing = 8;
  return launch_slope(s, GD_DTYPE_BF16, (cudaStream_t)stream) == cudaSuccess ? GD_OK : GD_ERR_CUDA;
}

}  // extern "C"
