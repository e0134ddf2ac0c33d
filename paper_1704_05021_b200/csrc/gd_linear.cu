// The linear layer (gd_linear_forward, gd_linear_backward): argument checks, the layout of ragged operands, the activation's
// slope with the bias gradient, and the products (gd_product_split.cu, gd_product_large.cu).
#include <algorithm>
#include <cmath>
#include <cstring>

#include "gd_mma.cuh"

namespace gd {

double cost_product_split(const Product& p);       // estimated cycles
cudaError_t launch_product_split(const Product& p, cudaStream_t stream);
cudaError_t launch_product_pair(const Product& p, cudaStream_t stream);

namespace {
// Estimated cycles of the pairs' kernel: 512 per k block of a 256 x 256 tile and what a tile costs besides, times the waves.
double cost_product_pair(const Product& p) {
  const double tiles = std::ceil(p.ep.rows / 256.0) * std::ceil(p.ep.cols / 256.0), blocks_k = std::ceil(p.depth / (double)kBlockK);
  return std::ceil(tiles / (sm_count() / 2)) * std::max(512.0 * blocks_k, 4000.0) + 6000.0;
}
}  // namespace

// Tiled-copy map of an operand.  The encoder is the driver's; it is asked for through the runtime, so that the library does not link
// against libcuda and loads on a machine without a GPU.
bool encode_tile(CUtensorMap* map, const void* p, uint64_t row_bytes, uint64_t width, uint64_t height, uint32_t box_width, uint32_t box_height, int dtype) {
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
  return reinterpret_cast<Encode>(f)(map, type, 2, const_cast<void*>(p), dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                     CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool encode_operand(CUtensorMap* map, const Operand& o, uint32_t extent, uint32_t depth, uint32_t box_extent, bool bf16) {
  return encode_tile(map, o.p, o.ld * 2, o.mn_major ? extent : depth, o.mn_major ? depth : extent, 64, box_extent, bf16 ? GD_DTYPE_BF16 : GD_DTYPE_FP16);
}
bool encode_piece(CUtensorMap* map, const void* p, uint64_t ld, const Epilogue& ep, int dtype) {
  const uint64_t item = dtype == GD_DTYPE_FP32 ? 4 : 2;
  return encode_tile(map, p, (ep.rows > 1 ? ld : (ep.cols + 7) / 8 * 8) * item, ep.cols, ep.rows, (uint32_t)(128 / item), 32, dtype);
}

cudaError_t launch_product(const Product& p, cudaStream_t stream) {
  if (p.ep.rows == 0 || p.ep.cols == 0) return cudaSuccess;
  ProfileScope ps(stream, PT_LINEAR);
  const bool pair = p.depth && cost_product_pair(p) < cost_product_split(p);
  const cudaError_t e = pair ? launch_product_pair(p, stream) : launch_product_split(p, stream);
  if (e == cudaSuccess) note_launches(1);
  return e;
}

namespace {

constexpr uint32_t kStatusBytes = 256;

// ---------------------------------------------------------------- ragged operands
// A matrix of 16-bit elements whose rows are no multiple of 16 bytes (or start anywhere), laid out with rows of ld_dst elements, a
// multiple of 8; the columns between are zeros.  A thread makes 16 bytes of the result: bound by the bytes, read and written once.
__global__ void __launch_bounds__(256) pack_kernel(const uint16_t* __restrict__ src, uint64_t ld, uint32_t rows, uint32_t cols, uint4* __restrict__ dst,
                                                   uint32_t vecs) {
  pdl_wait();
  pdl_trigger();
  const uint64_t total = (uint64_t)rows * vecs;
  for (uint64_t t = (uint64_t)blockIdx.x * 256u + threadIdx.x; t < total; t += (uint64_t)gridDim.x * 256u) {
    const uint32_t r = (uint32_t)(t / vecs), c = (uint32_t)(t % vecs) * 8u;
    const uint16_t* s = src + r * ld + c;
    uint32_t w[4];
    if (c + 8 <= cols && ((uintptr_t)s & 3u) == 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) w[j] = reinterpret_cast<const uint32_t*>(s)[j];
    } else {
#pragma unroll
      for (uint32_t j = 0; j < 4; ++j) {
        const uint32_t a = c + 2 * j < cols ? s[2 * j] : 0u, b = c + 2 * j + 1 < cols ? s[2 * j + 1] : 0u;
        w[j] = a | b << 16;
      }
    }
    dst[t] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}
cudaError_t launch_pack(const void* src, uint64_t ld, uint64_t rows, uint64_t cols, void* dst, cudaStream_t stream) {
  ProfileScope ps(stream, PT_LINEAR_PACK);
  const uint64_t vecs = (cols + 7) / 8, blocks = (rows * vecs + 255) / 256;
  const cudaError_t e = launch_dependent(pack_kernel, dim3((uint32_t)std::min<uint64_t>(blocks, (uint64_t)sm_count() * 16)), dim3(256), 0, stream,
                                         static_cast<const uint16_t*>(src), ld, (uint32_t)rows, (uint32_t)cols, static_cast<uint4*>(dst), (uint32_t)vecs);
  if (e == cudaSuccess) note_launches(1);
  return e;
}

// ---------------------------------------------------------------- dz and db
// dz = dy * act'(pre), rounded to the operands' type, and the sums of its columns before that rounding, in one pass over dy and pre.
// A cluster of kSlopeCtas CTAs takes 64 columns, each a share of the rows; a thread takes 8 neighbouring columns of every 32nd
// row.  The threads' sums meet in shared memory and the CTAs' through distributed shared memory, always in the same order: no atomics,
// no second launch.  Bound by the bytes (dy and pre read, dz written).
constexpr uint32_t kSlopeCtas = 8, kSlopeRows = 32;
struct SlopeArgs {
  const void* dy;
  const void* pre;
  void* dz;            // NULL: only the sums are wanted
  float* db;           // NULL: only dz is wanted
  uint64_t ld_dy, ld_pre, ld_dz;
  uint32_t rows, cols;
  int32_t activation;
  uint32_t accumulate, vectors;
};
template <int DT>
__global__ void __launch_bounds__(256) slope_kernel(const __grid_constant__ SlopeArgs a) {
  __shared__ float s_sum[kSlopeRows][64 + 1];
  __shared__ __align__(16) float s_total[64];
  pdl_wait();
  pdl_trigger();
  const uint32_t rank = cluster_rank(), tid = threadIdx.x, c = blockIdx.x / kSlopeCtas * 64u + (tid & 7u) * 8u;
  const uint32_t per = (a.rows + kSlopeCtas - 1) / kSlopeCtas, r0 = min(rank * per, a.rows), r1 = min(r0 + per, a.rows);
  const bool whole = a.vectors && c + 8 <= a.cols;
  float sum[8] = {};
  if (c < a.cols) {
#pragma unroll 2
    for (uint32_t r = r0 + (tid >> 3); r < r1; r += kSlopeRows) {
      float g[8], z[8];
      if (whole) {
        load8_as(a.dy, r * a.ld_dy + c, DT, g);
        if (a.activation != GD_ACT_NONE) load8_as(a.pre, r * a.ld_pre + c, DT, z);
      } else {
#pragma unroll
        for (uint32_t j = 0; j < 8; ++j) {
          const bool in = c + j < a.cols;
          g[j] = in ? load_as(a.dy, r * a.ld_dy + c + j, DT) : 0.f;
          z[j] = in && a.activation != GD_ACT_NONE ? load_as(a.pre, r * a.ld_pre + c + j, DT) : 0.f;
        }
      }
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (a.activation == GD_ACT_RELU) g[j] = z[j] > 0.f ? g[j] : 0.f * g[j];
        else if (a.activation == GD_ACT_GELU) g[j] *= gelu_slope(z[j]);
        else if (a.activation == GD_ACT_SILU) g[j] *= silu_slope(z[j]);
        sum[j] += g[j];
      }
      // (dz's own rows are padded to a multiple of 8 with zeros, which the ragged case above made)
      if (a.dz) store8_as(a.dz, r * a.ld_dz + c, DT, g);
    }
  }
  if (!a.db) return;
#pragma unroll
  for (int j = 0; j < 8; ++j) s_sum[tid >> 3][(tid & 7u) * 8u + j] = sum[j];
  __syncthreads();
  if (tid < 64) {
    float t = 0.f;
#pragma unroll 8
    for (uint32_t r = 0; r < kSlopeRows; ++r) t += s_sum[r][tid];
    s_total[tid] = t;
  }
  cluster_arrive();
  cluster_wait();
  const uint32_t col = blockIdx.x / kSlopeCtas * 64u + tid * 2u;
  if (rank == 0 && tid < 32) {
    float2 t = make_float2(0.f, 0.f);
    for (uint32_t q = 0; q < kSlopeCtas; ++q) {
      const float2 x = peer_load2(peer_address(smem_u32(s_total + 2 * tid), q));
      t.x += x.x, t.y += x.y;
    }
    if (col < a.cols) a.db[col] = a.accumulate ? a.db[col] + t.x : t.x;
    if (col + 1 < a.cols) a.db[col + 1] = a.accumulate ? a.db[col + 1] + t.y : t.y;
  }
  cluster_arrive();
  cluster_wait();
}
cudaError_t launch_slope(const SlopeArgs& a, int dtype, cudaStream_t stream) {
  ProfileScope ps(stream, PT_LINEAR_SLOPE);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((a.cols + 63) / 64 * kSlopeCtas);
  cfg.blockDim = dim3(256);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = kSlopeCtas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = dtype == GD_DTYPE_BF16 ? cudaLaunchKernelEx(&cfg, slope_kernel<GD_DTYPE_BF16>, a) : cudaLaunchKernelEx(&cfg, slope_kernel<GD_DTYPE_FP16>, a);
  if (e == cudaSuccess) note_launches(1);
  return e;
}

// ---------------------------------------------------------------- host side
uint64_t up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }
bool tiles_as_it_is(const void* p, uint64_t ld) { return aligned_to(p, 16) && ld % 8 == 0; }
// 16-byte accesses at columns that are multiples of 8 stay aligned
bool vector_rows(const void* p, uint64_t ld, int dt) { return !p || (aligned_to(p, 16) && ld * dtype_bytes(dt) % 16 == 0); }

struct Workspace {
  unsigned char* base;
  size_t at, size;
  void* take(uint64_t rows, uint64_t cols) {
    unsigned char* p = base + at;
    at += up(rows * up(cols, 8) * 2, 256);
    return at <= size ? p : nullptr;
  }
};
// A leading dimension for one row is never used: a ragged one would only cause a copy.
uint64_t row_step(uint64_t ld, uint64_t rows, uint64_t cols) { return rows > 1 ? ld : up(cols, 8); }

// `p` as an operand the tiled copies can read, laid out in the workspace if need be.
int operand(const void* p, uint64_t ld, uint64_t rows, uint64_t cols, Workspace& ws, cudaStream_t stream, Operand* o) {
  o->p = p;
  o->ld = row_step(ld, rows, cols);
  if (rows == 0 || cols == 0 || tiles_as_it_is(p, o->ld)) return GD_OK;
  void* q = ws.take(rows, cols);
  if (!q) return GD_ERR_WORKSPACE;
  if (launch_pack(p, ld, rows, cols, q, stream) != cudaSuccess) return GD_ERR_CUDA;
  o->p = q;
  o->ld = up(cols, 8);
  return GD_OK;
}
bool good_rows(const void* p, uint64_t ld, uint64_t rows, uint64_t cols, size_t item) {
  return p && aligned_to(p, item) && (rows <= 1 || ld >= cols) && !(ld >> 40);
}
int check_shape(uint64_t m, uint64_t n, uint64_t k, int dtype, int act, int layout) {
  if (!is_16bit(dtype) || act < GD_ACT_NONE || act > GD_ACT_SILU || (layout != GD_W_IN_OUT && layout != GD_W_OUT_IN)) return GD_ERR_INVALID_ARG;
  if (m >> 31 || n >> 31 || k >> 31) return GD_ERR_TOO_LARGE;
  return GD_OK;
}
int check_workspace(const void* ws, size_t bytes) { return !ws || !aligned_to(ws, 256) || bytes < kStatusBytes ? GD_ERR_WORKSPACE : GD_OK; }

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
  // (all sizes are known before anything is enqueued: a workspace that is too small is found here)
  {
    Workspace probe = ws;
    if (a->k && !tiles_as_it_is(a->x, row_step(a->ldx, a->m, a->k)) && !probe.take(a->m, a->k)) return GD_ERR_WORKSPACE;
    if (a->k && !tiles_as_it_is(a->w, row_step(a->ldw, w_rows, w_cols)) && !probe.take(w_rows, w_cols)) return GD_ERR_WORKSPACE;
  }
  Product p;
  std::memset(&p, 0, sizeof(p));
  if ((rc = operand(a->x, a->ldx, a->m, a->k, ws, stream, &p.a)) != GD_OK || (rc = operand(a->w, a->ldw, w_rows, w_cols, ws, stream, &p.b)) != GD_OK) return rc;
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
  return launch_product(p, stream) == cudaSuccess ? GD_OK : GD_ERR_CUDA;
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
  {
    Workspace probe = ws;
    if (has_dx && n && !tiles_as_it_is(a->w, row_step(a->ldw, w_rows, w_cols)) && !probe.take(w_rows, w_cols)) return GD_ERR_WORKSPACE;
    if (has_dw && m && !tiles_as_it_is(a->x, row_step(a->ldx, m, k)) && !probe.take(m, k)) return GD_ERR_WORKSPACE;
  }
  if (make || has_db) {
    s.dy = a->dy, s.ld_dy = a->ld_dy;
    s.pre = a->pre, s.ld_pre = a->ld_pre;
    s.db = has_db ? a->db : nullptr;
    s.rows = (uint32_t)m, s.cols = (uint32_t)n;
    s.activation = a->activation;
    s.accumulate = add;
    s.vectors = vector_rows(a->dy, row_step(a->ld_dy, m, n), a->dtype) && (!slope || vector_rows(a->pre, row_step(a->ld_pre, m, n), a->dtype));
    if (launch_slope(s, a->dtype, stream) != cudaSuccess) return GD_ERR_CUDA;
  }
  Product p;
  std::memset(&p, 0, sizeof(p));
  p.bf16 = a->dtype == GD_DTYPE_BF16;
  p.status = (int*)a->workspace;
  p.ep.dtype = a->dtype;
  if (has_dx) {                       // dx = dz W^T: contraction over n
    if (n && (rc = operand(a->w, a->ldw, w_rows, w_cols, ws, stream, &w)) != GD_OK) return rc;
    p.a = dz, p.a.mn_major = false;
    p.b = w, p.b.mn_major = !in_out;
    p.depth = (uint32_t)n;
    p.ep.out = a->dx, p.ep.ld_out = a->ld_dx, p.ep.out_dtype = a->dtype;
    p.ep.rows = (uint32_t)m, p.ep.cols = (uint32_t)k;
    p.ep.vectors = vector_rows(a->dx, row_step(a->ld_dx, m, k), a->dtype);
    if (launch_product(p, stream) != cudaSuccess) return GD_ERR_CUDA;
  }
  if (has_dw) {                       // dw = x^T dz, or its transpose: contraction over m
    if (m && (rc = operand(a->x, a->ldx, m, k, ws, stream, &x)) != GD_OK) return rc;
    p.a = in_out ? x : dz, p.b = in_out ? dz : x;
    p.a.mn_major = p.b.mn_major = true;
    p.depth = (uint32_t)m;
    p.ep.out = a->dw, p.ep.ld_out = a->ld_dw, p.ep.out_dtype = a->dw_dtype;
    p.ep.rows = (uint32_t)w_rows, p.ep.cols = (uint32_t)w_cols;
    if (add) p.ep.add = a->dw, p.ep.ld_add = a->ld_dw, p.ep.add_dtype = GD_DTYPE_FP32;
    p.ep.vectors = vector_rows(a->dw, row_step(a->ld_dw, w_rows, w_cols), a->dw_dtype);
    if (launch_product(p, stream) != cudaSuccess) return GD_ERR_CUDA;
  }
  return GD_OK;
}

}  // namespace
}  // namespace gd

extern "C" {

int gd_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, int any_layout, size_t* bytes_out) {
  using namespace gd;
  if (!bytes_out) return GD_ERR_INVALID_ARG;
  if (m >> 31 || n >> 31 || k >> 31) return GD_ERR_TOO_LARGE;
  auto matrix = [](uint64_t rows, uint64_t cols) { return up(rows * up(cols, 8) * 2, 256); };
  uint64_t b = kStatusBytes + matrix(m, n);                              // dz
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

int gd_linear_forward(const gd_linear_forward_args* a, void* stream) { return gd::forward(a, (cudaStream_t)stream); }

int gd_linear_backward(const gd_linear_backward_args* a, void* stream) { return gd::backward(a, (cudaStream_t)stream); }

}  // extern "C"
