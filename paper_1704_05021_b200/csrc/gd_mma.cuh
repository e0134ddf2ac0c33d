// Tensor-core products on sm_100a: tiled copies into swizzled shared memory, tcgen05.mma with accumulators in tensor
// memory, and the epilogue the linear layer's kernels share.
//
// The products are D[i, j] = sum_k A(i, k) B(j, k) with 16-bit operands.  Shared memory holds a block of 64 k in rows of 128
// bytes under the 128-byte swizzle (the hardware XORs address bits 4..6 with bits 7..9), in one of two forms:
//   K-major   rows are i (or j), 64 consecutive k in a row: one copy box {64 k, rows}
//   MN-major  rows are k, 64 consecutive i (or j) in a row: boxes {64 i, 64 k} of 8 KB, one per 64 i
// so an operand is read as it lies in memory, transposed or not.
#pragma once

#include <cuda.h>      // CUtensorMap (types only: the encoder is asked from the runtime)

#include "gd_train.cuh"

namespace gd {

constexpr uint32_t kBlockK = 64;

// ---------------------------------------------------------------- clusters
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// (the .aligned forms want the whole warp: it is brought together first.  Only launches with a cluster dimension execute these, mapa or
// st.async: without one an st.async to the CTA itself ended in an illegal instruction.)
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive_relaxed() {      // publishes nothing
  __syncwarp();
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t peer_address(uint32_t smem_address, uint32_t rank) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_address), "r"(rank));
  return a;
}
__device__ __forceinline__ float4 peer_load4(uint32_t a) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float peer_load1(uint32_t a) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ float2 peer_load2(uint32_t a) {
  float2 v;
  asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a) : "memory");
  return v;
}

// Eight bytes into a CTA of the cluster, counted on an mbarrier there.
__device__ __forceinline__ void send_peer2(uint32_t address, float2 v, uint32_t barrier) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(address), "f"(v.x), "f"(v.y), "r"(barrier) : "memory");
}

// True in one thread of the (converged) warp, the same one every time.  The instructions that ask for copies and products take their operands from registers of
// the whole warp; behind a branch on this the compiler knows that one thread is left and issues them directly.
__device__ __forceinline__ bool elect_one() {
  uint32_t p;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
  return p != 0u;
}

// ---------------------------------------------------------------- copies and products
__device__ __forceinline__ void tile_load(void* dst, const CUtensorMap* map, int32_t x, int32_t y, uint64_t* b) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
               "l"(map), "r"(x), "r"(y), "r"(smem_u32(b))
               : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }

// Shared-memory descriptor of an operand block (128-byte swizzle; bit 46: the sm_100 form).  The stride between groups of 8 rows
// is 1024 bytes in both forms; `lead` is the distance between boxes of 64 i (MN-major; not used K-major).
__device__ __forceinline__ uint64_t operand_desc(uint32_t smem_address, uint32_t lead) {
  return (uint64_t)((smem_address & 0x3FFFFu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// Instruction descriptor: fp32 accumulators, both operands bf16 or both fp16.
__host__ __device__ constexpr uint32_t mma_desc(uint32_t m, uint32_t n, bool bf16, bool a_mn, bool b_mn) {
  return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (a_mn ? 1u : 0u) << 15 | (b_mn ? 1u : 0u) << 16 | (n >> 3) << 17 | (m >> 4) << 24;
}
template <int CTAS>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, bool add) {
  if constexpr (CTAS == 1)
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                 "r"(desc), "r"((uint32_t)add)
                 : "memory");
  else
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
                 "r"(desc), "r"((uint32_t)add)
                 : "memory");
}
// b receives one arrive when all products issued so far by this thread have been done.
__device__ __forceinline__ void mma_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
template <int CTAS>
__device__ __forceinline__ void tmem_alloc(uint32_t* dst, uint32_t columns) {
  if constexpr (CTAS == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst)), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
}
template <int CTAS>
__device__ __forceinline__ void tmem_free(uint32_t address, uint32_t columns) {
  if constexpr (CTAS == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(address), "r"(columns) : "memory");
}
// Eight columns of the warp's 32 accumulator lanes: r[c] of lane l is D[l, c].  tmem_ready() before the registers are used.
__device__ __forceinline__ void tmem_load8(uint32_t address, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7])
               : "r"(address)
               : "memory");
}
// Thirty-two columns, one instruction.
__device__ __forceinline__ void tmem_load32(uint32_t address, float* r) {
  uint32_t* u = reinterpret_cast<uint32_t*>(r);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, %20, %21, %22, "
      "%23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]),
        "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]),
        "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
      : "r"(address)
      : "memory");
}
__device__ __forceinline__ void tmem_ready() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// ---------------------------------------------------------------- activations and epilogue
// x Phi(x) and x / (1 + exp(-x)), and their slopes.  Phi by formula 7.1.26 of Abramowitz and Stegun (erf to 1.5e-7, one
// exponential that is also the density's): a third of the instructions of erff, which a tile's 65536 values pay for.
__device__ __forceinline__ float normal_cdf(float x, float* gauss) {
  const float a = fabsf(x) * 0.70710678118654752f;
  const float t = __fdividef(1.f, fmaf(0.3275911f, a, 1.f));
  const float e = __expf(-a * a);
  float p = fmaf(1.061405429f, t, -1.453152027f);
  p = fmaf(p, t, 1.421413741f);
  p = fmaf(p, t, -0.284496736f);
  p = fmaf(p, t, 0.254829592f);
  const float tail = 0.5f * p * t * e;
  *gauss = e;
  return x < 0.f ? tail : 1.f - tail;
}
__device__ __forceinline__ float gelu(float x) {
  float e;
  return x * normal_cdf(x, &e);
}
__device__ __forceinline__ float gelu_slope(float x) {
  float e;
  const float phi = normal_cdf(x, &e);
  return fmaf(x * 0.39894228040143268f, e, phi);
}
__device__ __forceinline__ float silu(float x) { return __fdividef(x, 1.f + __expf(-x)); }
__device__ __forceinline__ float silu_slope(float x) {
  const float s = __fdividef(1.f, 1.f + __expf(-x));
  return s * (1.f + x * (1.f - s));
}
__device__ __forceinline__ float activate(float z, int act) {
  switch (act) {
    case GD_ACT_RELU: return z < 0.f ? 0.f : z;      // (a NaN stays one)
    case GD_ACT_GELU: return gelu(z);
    case GD_ACT_SILU: return silu(z);
    default: return z;
  }
}

// What happens to a product on its way out: out[r, c] = act(D + bias[c]) + add[r, c], and pre[r, c] = D + bias[c].
struct Epilogue {
  void* out;
  const void* bias;
  const void* add;
  void* pre;
  uint64_t ld_out, ld_add, ld_pre;
  uint32_t rows, cols;
  int32_t dtype;        // of pre (16 bits)
  int32_t out_dtype, bias_dtype, add_dtype;
  int32_t activation;
  uint32_t vectors;     // every buffer above takes 16-byte accesses at columns that are multiples of 8
  uint32_t pairs;       // out, add and pre are of 16 bits and take 4-byte accesses at even columns
};

__device__ __forceinline__ float load_as(const void* p, uint64_t i, int dt) {
  if (dt == GD_DTYPE_FP32) return static_cast<const float*>(p)[i];
  return dt == GD_DTYPE_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]) : __half2float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, uint64_t i, int dt, float x) {
  if (dt == GD_DTYPE_FP32) static_cast<float*>(p)[i] = x;
  else if (dt == GD_DTYPE_BF16) static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(x);
  else static_cast<__half*>(p)[i] = __float2half_rn(x);
}
// (one branch for all eight, not one per pair: the code between branches is what the instruction caches see)
template <int DT>
__device__ __forceinline__ void widen8_t(const uint4& q, float (&x)[8]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const float2 f = unpack2<DT>(w[j]);
    x[2 * j] = f.x, x[2 * j + 1] = f.y;
  }
}
__device__ __forceinline__ void widen8(const uint4& q, int dt, float (&x)[8]) {
  if (dt == GD_DTYPE_BF16) widen8_t<GD_DTYPE_BF16>(q, x); else widen8_t<GD_DTYPE_FP16>(q, x);
}
template <int DT>
__device__ __forceinline__ uint4 narrow8_t(const float* x) {
  return make_uint4(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]), pack2<DT>(x[4], x[5]), pack2<DT>(x[6], x[7]));
}
__device__ __forceinline__ uint4 narrow8(const float* x, int dt) { return dt == GD_DTYPE_BF16 ? narrow8_t<GD_DTYPE_BF16>(x) : narrow8_t<GD_DTYPE_FP16>(x); }
__device__ __forceinline__ void load8_as(const void* p, uint64_t i, int dt, float (&x)[8]) {
  if (dt == GD_DTYPE_FP32) {
    const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(p) + i);
    const float4 a = q[0], b = q[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
    return;
  }
  widen8(*reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + i), dt, x);
}
__device__ __forceinline__ void store8_as(void* p, uint64_t i, int dt, const float (&x)[8]) {
  if (dt == GD_DTYPE_FP32) {
    float4* q = reinterpret_cast<float4*>(static_cast<float*>(p) + i);
    q[0] = make_float4(x[0], x[1], x[2], x[3]);
    q[1] = make_float4(x[4], x[5], x[6], x[7]);
    return;
  }
  *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + i) = narrow8(x, dt);
}
template <int N>
__device__ __forceinline__ void activate_all(float* v, int act) {
  if (act == GD_ACT_RELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = v[j] < 0.f ? 0.f : v[j];
  } else if (act == GD_ACT_GELU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = gelu(v[j]);
  } else if (act == GD_ACT_SILU) {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = silu(v[j]);
  }
}
// Up to eight elements of one output column, from row r on, z = D + bias given.
__device__ __forceinline__ void finish_column(const Epilogue& e, uint32_t r, uint32_t c, float (&z)[8], uint32_t most = 8) {
  const uint32_t rows = min(e.rows - min(r, e.rows), most);
  const uint64_t at = (uint64_t)r * e.ld_out + c;
  if (e.pre) {
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u)
      if (u < rows) store_as(e.pre, (uint64_t)(r + u) * e.ld_pre + c, e.dtype, z[u]);
  }
  activate_all<8>(z, e.activation);
  if (e.add) {
    float w[8];
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) w[u] = u < rows ? load_as(e.add, (uint64_t)(r + u) * e.ld_add + c, e.add_dtype) : 0.f;
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) z[u] += w[u];
  }
  if (e.out_dtype == GD_DTYPE_FP32) {
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u)
      if (u < rows) static_cast<float*>(e.out)[at + u * e.ld_out] = z[u];
  } else {
    const bool bf16 = e.out_dtype == GD_DTYPE_BF16;
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) {
      const uint32_t w = bf16 ? pack2<GD_DTYPE_BF16>(z[u], 0.f) : pack2<GD_DTYPE_FP16>(z[u], 0.f);
      if (u < rows) static_cast<uint16_t*>(e.out)[at + u * e.ld_out] = (uint16_t)w;
    }
  }
}
// The same of columns c and c + 1, c even, where e.pairs holds: one access for both (c may be the last column).
__device__ __forceinline__ void finish_columns(const Epilogue& e, uint32_t r, uint32_t c, float (&z)[8], float (&y)[8], uint32_t most = 8) {
  const uint32_t rows = min(e.rows - min(r, e.rows), most);
  const bool bf16 = e.out_dtype == GD_DTYPE_BF16, both = c + 1 < e.cols;      // (the type of all three)
  const auto put = [&](void* to, uint64_t ld) {
    uint16_t* at = static_cast<uint16_t*>(to) + (uint64_t)r * ld + c;
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) {
      const uint32_t w = bf16 ? pack2<GD_DTYPE_BF16>(z[u], y[u]) : pack2<GD_DTYPE_FP16>(z[u], y[u]);
      if (u < rows && both) *reinterpret_cast<uint32_t*>(at + u * ld) = w;
      if (u < rows && !both) at[u * ld] = (uint16_t)w;
    }
  };
  if (e.pre) put(e.pre, e.ld_pre);
  activate_all<8>(z, e.activation);
  activate_all<8>(y, e.activation);
  if (e.add) {
    const uint16_t* at = static_cast<const uint16_t*>(e.add) + (uint64_t)r * e.ld_add + c;
    uint32_t w[8];
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) w[u] = u < rows ? (both ? *reinterpret_cast<const uint32_t*>(at + u * e.ld_add) : at[u * e.ld_add]) : 0u;
#pragma unroll
    for (uint32_t u = 0; u < 8; ++u) {
      const float2 f = bf16 ? unpack2<GD_DTYPE_BF16>(w[u]) : unpack2<GD_DTYPE_FP16>(w[u]);
      z[u] += f.x, y[u] += f.y;
    }
  }
  put(e.out, e.ld_out);
}
// Eight neighbours of one output row, c a multiple of 8.
__device__ __forceinline__ void finish8(const Epilogue& e, uint32_t r, uint32_t c, float (&v)[8]) {
  if (r >= e.rows || c >= e.cols) return;
  if (e.vectors && c + 8 <= e.cols) {
    if (e.bias) {
      float b[8];
      load8_as(e.bias, c, e.bias_dtype, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += b[j];
    }
    if (e.pre) store8_as(e.pre, (uint64_t)r * e.ld_pre + c, e.dtype, v);
    activate_all<8>(v, e.activation);
    if (e.add) {
      float b[8];
      load8_as(e.add, (uint64_t)r * e.ld_add + c, e.add_dtype, b);
#pragma unroll
      for (int j = 0; j < 8; ++j) v[j] += b[j];
    }
    store8_as(e.out, (uint64_t)r * e.ld_out + c, e.out_dtype, v);
    return;
  }
#pragma unroll
  for (uint32_t j = 0; j < 8; ++j) {
    if (c + j >= e.cols) break;
    float z = e.bias ? v[j] + load_as(e.bias, c + j, e.bias_dtype) : v[j];
    if (e.pre) store_as(e.pre, (uint64_t)r * e.ld_pre + c + j, e.dtype, z);
    z = activate(z, e.activation);
    if (e.add) z += load_as(e.add, (uint64_t)r * e.ld_add + c + j, e.add_dtype);
    store_as(e.out, (uint64_t)r * e.ld_out + c + j, e.out_dtype, z);
  }
}

// ---------------------------------------------------------------- host side
// A 16-bit matrix whose rows are contiguous, as one operand: `extent` values of i (or j) and `depth` of k.
struct Operand {
  const void* p;
  uint64_t ld;
  bool mn_major;       // rows of the matrix are k
};
struct Product {
  Operand a, b;        // of the output's rows and of its columns
  uint32_t depth;      // extent of k
  bool bf16;
  Epilogue ep;
  int* status;
  float* partial;      // kPartialBytes of workspace where the depth is at least kLongDepth, else NULL
  // The launch before this one in the stream is a product too, waits for all before it, and neither touches what the other writes: this one
  // runs on the SMs that the other leaves idle in its last wave (pdl_wait stands at its end, so that whatever follows has both).
  bool beside;
  bool followed;       // the launch after this one is such a product: what this one's last wave leaves idle is no loss
};
constexpr uint64_t kLongDepth = 16384, kPartialBytes = 2u << 20;
// How many k blocks the tensor cores may sum in one go.  Their fp32 accumulator truncates: measured against 64 bits the relative
// error of a product of normal numbers grows by 1.1e-9 per k (4.4e-6 at 4096, where fp32 additions in registers leave 6e-7).
// Next to the 2^-9 of a 16-bit result that is nothing; an fp32 result is summed in chains of 512 k (5e-7) that are joined in
// registers, rounded to nearest.
constexpr uint32_t kChainBlocks = 512 / kBlockK;
inline uint32_t chain_blocks(const Product& p) { return p.ep.out_dtype == GD_DTYPE_FP32 ? kChainBlocks : 0x7FFFFFFFu; }
bool encode_operand(CUtensorMap* map, const Operand& o, uint32_t extent, uint32_t depth, uint32_t box_extent, bool bf16);
struct SplitChoice {       // of the split kernel's tile
  bool transposed;         // D's lanes are the output's columns
  uint32_t bn, splits;
  uint32_t outer;          // parts of k in clusters of their own, joined by a second launch
  double cost;             // estimated cycles
};
bool encode_piece(CUtensorMap* map, const void* p, uint64_t ld, const Epilogue& ep, uint32_t cols, int dtype);     // 32 rows x 128 bytes of a result, up to `cols`
cudaError_t launch_product(const Product& p, cudaStream_t stream);

}  // namespace gd
