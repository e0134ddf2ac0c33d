// One AdamW update of many tensors (gd_adamw_step): a stream over parameters, gradients and moments.
//
// The update is elementwise, so the bytes bound it: 28 per element with fp32 throughout, 16.1 with the moments in
// 8 bits.  One launch takes up to kMaxTensors tensors, whose table travels as the kernel argument (no device copy, no
// allocation); a CTA takes one chunk of kChunk consecutive elements of one tensor.  A warp works on blocks of 128 elements, four
// per lane in one 16-byte access, because 128 is also the unit that shares a scale in the 8-bit moments: its largest
// magnitude is one warp reduction, and nothing but the warp has to agree on it.  kBlocks of them are in flight per warp.
// A tensor whose buffers do not all start on a vector boundary (pieces of a flat vector do not), and a tensor's last,
// partial block, go element by element, lane-contiguous, with the same arithmetic.
#include <cmath>

#include "gd_train.cuh"

namespace gd {
namespace {

constexpr int kBlocks = 2;                        // blocks of 128 elements a warp has in flight
constexpr uint32_t kAdamThreads = 256;
constexpr uint32_t kChunk = kAdamThreads / 32 * kBlocks * 128;

struct TensorEntry {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  uint64_t n;
  uint32_t chunk0;      // first chunk of the tensor in this launch
  uint32_t index;       // its place in the call's list (enters the random numbers)
  float decay;          // 1 - lr * weight_decay
  uint32_t vectors;     // all buffers start on a boundary of four elements
};

struct AdamScalars {
  float beta1, one_minus_beta1, beta2, one_minus_beta2, root_factor, eps, step_size, grad_scale;
  const float* grad_scale_dev;
  uint32_t seed;
  uint32_t n_tensors;
  int32_t copy_dtype;
};

// Kernel arguments hold at most 32764 bytes.  The short table is for the usual model: a launch pays for its argument's bytes.
constexpr uint32_t kFewTensors = 24, kMaxTensors = 400;
template <uint32_t CAP>
struct AdamTable {
  AdamScalars s;
  TensorEntry t[CAP];
};
static_assert(sizeof(AdamTable<kMaxTensors>) <= 32764, "a kernel argument");

template <int DT>
__device__ __forceinline__ void load4(const void* base, uint64_t at, float (&x)[4]) {
  if constexpr (DT == GD_DTYPE_FP32) {
    const float4 q = __ldcs(reinterpret_cast<const float4*>(static_cast<const float*>(base) + at));
    x[0] = q.x, x[1] = q.y, x[2] = q.z, x[3] = q.w;
  } else {
    const uint2 q = __ldcs(reinterpret_cast<const uint2*>(static_cast<const uint16_t*>(base) + at));
    const float2 a = unpack2<DT>(q.x), b = unpack2<DT>(q.y);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  }
}
template <int DT>
__device__ __forceinline__ void store4(void* base, uint64_t at, const float (&x)[4]) {
  if constexpr (DT == GD_DTYPE_FP32)
    __stcs(reinterpret_cast<float4*>(static_cast<float*>(base) + at), make_float4(x[0], x[1], x[2], x[3]));
  else
    __stcs(reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + at), make_uint2(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3])));
}
template <int DT>
__device__ __forceinline__ float load1(const void* base, uint64_t at) {
  return Elem<DT>::get(static_cast<const typename Elem<DT>::type*>(base)[at]);
}
template <int DT>
__device__ __forceinline__ void store1(void* base, uint64_t at, float x) {
  static_cast<typename Elem<DT>::type*>(base)[at] = Elem<DT>::put(x);
}

__device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7FEB352Du;
  x ^= x >> 15;
  x *= 0x846CA68Bu;
  return x ^ (x >> 16);
}

// fp8 (e4m3) of a magnitude y < 256, rounded up or down by 16 random bits.  In units of the last bit kept, times 2^20, a normal
// number is its own bits less the exponent's bias; below 2^-6 the step is fixed, which adding 2^-6 turns into the same form.
__device__ __forceinline__ uint32_t encode_fp8(float y, uint32_t random16) {
  const uint32_t units = y >= 0x1p-6f ? __float_as_uint(y) - (120u << 23) : __float_as_uint(__fadd_rn(y, 0x1p-6f)) - (121u << 23);
  const uint32_t code = (units + (random16 << 4)) >> 20;
  return (__float_as_uint(y) & 0x7F800000u) == 0x7F800000u ? 127u : min(code, 127u);
}
__device__ __forceinline__ float2 decode_fp8x2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// The scale of a block from the bits of its largest magnitude, and its reciprocal: powers of two, so both products are exact.
__device__ __forceinline__ void block_scale(uint32_t top_bits, float* scale, float* inverse) {
  const int e = max((int)(top_bits >> 23) - 7, 1);
  *scale = __uint_as_float((uint32_t)e << 23);
  *inverse = __uint_as_float((uint32_t)(254 - e) << 23);
}

// the update in the order the header states; nothing may be contracted into a fused multiply-add
__device__ __forceinline__ void update(float& p, float g, float& m, float& v, float& root, const AdamScalars& s, float scale, float decay) {
  g = __fmul_rn(g, scale);
  m = __fadd_rn(__fmul_rn(m, s.beta1), __fmul_rn(g, s.one_minus_beta1));
  v = __fadd_rn(__fmul_rn(v, s.beta2), __fmul_rn(__fmul_rn(g, s.one_minus_beta2), g));
  root = __fsqrt_rn(v);
  const float d = __fadd_rn(__fmul_rn(root, s.root_factor), s.eps);
  p = __fsub_rn(__fmul_rn(p, decay), __fmul_rn(__fdiv_rn(m, d), s.step_size));
}

template <int PT, int GT, int BITS, uint32_t CAP>
__global__ void __launch_bounds__(kAdamThreads) adamw_kernel(const __grid_constant__ AdamTable<CAP> table) {
  const AdamScalars& s = table.s;
  // the tensor this chunk belongs to
  uint32_t lo = 0, hi = s.n_tensors;
  while (hi - lo > 1) {
    const uint32_t mid = (lo + hi) >> 1;
    if (table.t[mid].chunk0 <= blockIdx.x) lo = mid; else hi = mid;
  }
  const TensorEntry& t = table.t[lo];
  const uint32_t lane = lane_id();
  const uint64_t first = (uint64_t)(blockIdx.x - t.chunk0) * kChunk + (threadIdx.x >> 5) * (kBlocks * 128u);
  const uint64_t n = t.n;
  if (first >= n) return;
  pdl_wait();
  pdl_trigger();
  const float scale = s.grad_scale_dev ? __fmul_rn(s.grad_scale, *s.grad_scale_dev) : s.grad_scale;
  const bool vec = t.vectors && first + kBlocks * 128u <= n;

  float p[kBlocks][4], g[kBlocks][4], m[kBlocks][4], v[kBlocks][4];
  uint32_t mc[kBlocks], vc[kBlocks];
  float ms[kBlocks], vs[kBlocks];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const uint64_t at = first + b * 128u;
    if (vec) {
      load4<PT>(t.param, at + 4 * lane, p[b]);
      load4<GT>(t.grad, at + 4 * lane, g[b]);
      if constexpr (BITS == 32) {
        load4<GD_DTYPE_FP32>(t.m, at + 4 * lane, m[b]);
        load4<GD_DTYPE_FP32>(t.v, at + 4 * lane, v[b]);
      } else {
        mc[b] = __ldcs(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.m) + at + 4 * lane));
        vc[b] = __ldcs(reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(t.v) + at + 4 * lane));
        ms[b] = t.m_scale[at >> 7];
        vs[b] = t.v_scale[at >> 7];
      }
    } else {
      mc[b] = vc[b] = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t e = at + lane + 32 * j;
        const bool in = e < n;
        p[b][j] = in ? load1<PT>(t.param, e) : 0.f;
        g[b][j] = in ? load1<GT>(t.grad, e) : 0.f;
        if constexpr (BITS == 32) {
          m[b][j] = in ? static_cast<const float*>(t.m)[e] : 0.f;
          v[b][j] = in ? static_cast<const float*>(t.v)[e] : 0.f;
        } else if (in) {
          mc[b] |= (uint32_t)static_cast<const uint8_t*>(t.m)[e] << (8 * j);
          vc[b] |= (uint32_t)static_cast<const uint8_t*>(t.v)[e] << (8 * j);
        }
      }
      if constexpr (BITS == 8) {
        ms[b] = at < n ? t.m_scale[at >> 7] : 0.f;
        vs[b] = at < n ? t.v_scale[at >> 7] : 0.f;
      }
    }
  }
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
    const uint64_t at = first + b * 128u;
    if (at >= n) break;
    float root[4];
    if constexpr (BITS == 8) {
      const float2 m01 = decode_fp8x2(mc[b] & 0xFFFFu), m23 = decode_fp8x2(mc[b] >> 16);
      const float2 v01 = decode_fp8x2(vc[b] & 0xFFFFu), v23 = decode_fp8x2(vc[b] >> 16);
      m[b][0] = __fmul_rn(m01.x, ms[b]), m[b][1] = __fmul_rn(m01.y, ms[b]), m[b][2] = __fmul_rn(m23.x, ms[b]), m[b][3] = __fmul_rn(m23.y, ms[b]);
      const float r[4] = {__fmul_rn(v01.x, vs[b]), __fmul_rn(v01.y, vs[b]), __fmul_rn(v23.x, vs[b]), __fmul_rn(v23.y, vs[b])};
#pragma unroll
      for (int j = 0; j < 4; ++j) v[b][j] = __fmul_rn(r[j], r[j]);
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) update(p[b][j], g[b][j], m[b][j], v[b][j], root[j], s, scale, t.decay);
    if constexpr (BITS == 8) {
      uint32_t m_top = 0u, v_top = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const bool in = vec || at + lane + 32 * j < n;      // (elements past the end hold zeros, but eps = 0 would make them NaN in p only)
        m_top = max(m_top, in ? __float_as_uint(m[b][j]) & 0x7FFFFFFFu : 0u);
        v_top = max(v_top, in ? __float_as_uint(root[j]) & 0x7FFFFFFFu : 0u);
      }
      m_top = __reduce_max_sync(0xFFFFFFFFu, m_top);
      v_top = __reduce_max_sync(0xFFFFFFFFu, v_top);
      float m_scale, m_inverse, v_scale, v_inverse;
      block_scale(m_top, &m_scale, &m_inverse);
      block_scale(v_top, &v_scale, &v_inverse);
      mc[b] = vc[b] = 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t e = (uint32_t)at + (vec ? 4 * lane + j : lane + 32 * j);
        const uint32_t h = mix32(e * 0x9E3779B9u + s.seed + t.index * 0x85EBCA77u);
        const uint32_t sign = __float_as_uint(m[b][j]) >> 31 << 7;
        const uint32_t cm = encode_fp8(__fmul_rn(fabsf(m[b][j]), m_inverse), h >> 16) | sign;
        uint32_t cv = encode_fp8(__fmul_rn(fabsf(root[j]), v_inverse), h & 0xFFFFu);
        if (root[j] > 0.f && cv == 0u) cv = 1u;
        cv |= __float_as_uint(root[j]) >> 31 << 7;
        mc[b] |= cm << (8 * j);
        vc[b] |= cv << (8 * j);
      }
      if (lane == 0) {
        t.m_scale[at >> 7] = m_scale;
        t.v_scale[at >> 7] = v_scale;
      }
    }
    if (vec) {
      store4<PT>(t.param, at + 4 * lane, p[b]);
      if (t.copy) {
        if (s.copy_dtype == GD_DTYPE_BF16) store4<GD_DTYPE_BF16>(t.copy, at + 4 * lane, p[b]);
        else if (s.copy_dtype == GD_DTYPE_FP16) store4<GD_DTYPE_FP16>(t.copy, at + 4 * lane, p[b]);
        else store4<GD_DTYPE_FP32>(t.copy, at + 4 * lane, p[b]);
      }
      if constexpr (BITS == 32) {
        store4<GD_DTYPE_FP32>(t.m, at + 4 * lane, m[b]);
        store4<GD_DTYPE_FP32>(t.v, at + 4 * lane, v[b]);
      } else {
        __stcs(reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.m) + at + 4 * lane), mc[b]);
        __stcs(reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + at + 4 * lane), vc[b]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t e = at + lane + 32 * j;
        if (e >= n) continue;
        store1<PT>(t.param, e, p[b][j]);
        if (t.copy) {
          if (s.copy_dtype == GD_DTYPE_BF16) store1<GD_DTYPE_BF16>(t.copy, e, p[b][j]);
          else if (s.copy_dtype == GD_DTYPE_FP16) store1<GD_DTYPE_FP16>(t.copy, e, p[b][j]);
          else store1<GD_DTYPE_FP32>(t.copy, e, p[b][j]);
        }
        if constexpr (BITS == 32) {
          static_cast<float*>(t.m)[e] = m[b][j];
          static_cast<float*>(t.v)[e] = v[b][j];
        } else {
          static_cast<uint8_t*>(t.m)[e] = (uint8_t)(mc[b] >> (8 * j));
          static_cast<uint8_t*>(t.v)[e] = (uint8_t)(vc[b] >> (8 * j));
        }
      }
    }
  }
}

template <int PT, int GT, int BITS>
cudaError_t launch_cap(const AdamTable<kMaxTensors>& full, uint32_t chunks, cudaStream_t stream) {
  if (full.s.n_tensors <= kFewTensors) {
    AdamTable<kFewTensors> few;
    few.s = full.s;
    for (uint32_t i = 0; i < full.s.n_tensors; ++i) few.t[i] = full.t[i];
    return launch_dependent(adamw_kernel<PT, GT, BITS, kFewTensors>, dim3(chunks), dim3(kAdamThreads), 0, stream, few);
  }
  return launch_dependent(adamw_kernel<PT, GT, BITS, kMaxTensors>, dim3(chunks), dim3(kAdamThreads), 0, stream, full);
}
template <int PT, int GT>
cudaError_t launch_bits(int bits, const AdamTable<kMaxTensors>& table, uint32_t chunks, cudaStream_t stream) {
  return bits == 8 ? launch_cap<PT, GT, 8>(table, chunks, stream) : launch_cap<PT, GT, 32>(table, chunks, stream);
}
template <int PT>
cudaError_t launch_grad(int gt, int bits, const AdamTable<kMaxTensors>& table, uint32_t chunks, cudaStream_t stream) {
  switch (gt) {
    case GD_DTYPE_FP32: return launch_bits<PT, GD_DTYPE_FP32>(bits, table, chunks, stream);
    case GD_DTYPE_BF16: return launch_bits<PT, GD_DTYPE_BF16>(bits, table, chunks, stream);
    default: return launch_bits<PT, GD_DTYPE_FP16>(bits, table, chunks, stream);
  }
}
cudaError_t launch_adamw(int pt, int gt, int bits, const AdamTable<kMaxTensors>& table, uint32_t chunks, cudaStream_t stream) {
  ProfileScope ps(stream, PT_ADAMW);
  cudaError_t e;
  switch (pt) {
    case GD_DTYPE_FP32: e = launch_grad<GD_DTYPE_FP32>(gt, bits, table, chunks, stream); break;
    case GD_DTYPE_BF16: e = launch_grad<GD_DTYPE_BF16>(gt, bits, table, chunks, stream); break;
    default: e = launch_grad<GD_DTYPE_FP16>(gt, bits, table, chunks, stream); break;
  }
  if (e == cudaSuccess) note_launches(1);
  return e;
}

}  // namespace
}  // namespace gd

extern "C" int gd_adamw_step(const gd_adamw_args* a, void* stream) {
  using namespace gd;
  if (!a || a->reserved != 0 || (a->n_tensors && !a->tensors)) return GD_ERR_INVALID_ARG;
  if (a->state_bits != 8 && a->state_bits != 32) return GD_ERR_INVALID_ARG;
  if (!is_dtype(a->param_dtype) || !is_dtype(a->grad_dtype) || !is_dtype(a->copy_dtype)) return GD_ERR_INVALID_ARG;
  if (a->step == 0 || !std::isfinite(a->lr) || !std::isfinite(a->eps) || !(a->eps >= 0.0)) return GD_ERR_INVALID_ARG;
  if (!(a->beta1 >= 0.0 && a->beta1 < 1.0 && a->beta2 >= 0.0 && a->beta2 < 1.0)) return GD_ERR_INVALID_ARG;
  if (!aligned_to(a->grad_scale_dev, 4)) return GD_ERR_INVALID_ARG;
  const bool eight = a->state_bits == 8;
  const size_t pb = dtype_bytes(a->param_dtype), gb = dtype_bytes(a->grad_dtype), cb = dtype_bytes(a->copy_dtype), sb = eight ? 1 : 4;
  for (uint32_t i = 0; i < a->n_tensors; ++i) {
    const gd_adamw_tensor& t = a->tensors[i];
    if (!std::isfinite(t.weight_decay)) return GD_ERR_INVALID_ARG;
    if (t.n == 0) continue;
    if (t.n >> 40) return GD_ERR_TOO_LARGE;
    if (!t.param || !t.grad || !t.m || !t.v || (eight && (!t.m_scale || !t.v_scale))) return GD_ERR_INVALID_ARG;
    if (!aligned_to(t.param, pb) || !aligned_to(t.grad, gb) || !aligned_to(t.m, sb) || !aligned_to(t.v, sb) || !aligned_to(t.copy, cb))
      return GD_ERR_INVALID_ARG;
    if (eight && (!aligned_to(t.m_scale, 4) || !aligned_to(t.v_scale, 4))) return GD_ERR_INVALID_ARG;
  }
  AdamTable<kMaxTensors> table;
  AdamScalars& s = table.s;
  s.beta1 = (float)a->beta1;
  s.one_minus_beta1 = (float)(1.0 - a->beta1);
  s.beta2 = (float)a->beta2;
  s.one_minus_beta2 = (float)(1.0 - a->beta2);
  s.root_factor = (float)(1.0 / std::sqrt(1.0 - std::pow(a->beta2, (double)a->step)));
  s.eps = (float)a->eps;
  s.step_size = (float)(a->lr / (1.0 - std::pow(a->beta1, (double)a->step)));
  s.grad_scale = a->grad_scale;
  s.grad_scale_dev = a->grad_scale_dev;
  s.seed = a->seed;
  s.copy_dtype = a->copy_dtype;
  s.n_tensors = 0;
  uint64_t chunks = 0;
  auto flush = [&]() -> int {
    if (s.n_tensors == 0) return GD_OK;
    const cudaError_t e = launch_adamw(a->param_dtype, a->grad_dtype, a->state_bits, table, (uint32_t)chunks, (cudaStream_t)stream);
    s.n_tensors = 0;
    chunks = 0;
    return e == cudaSuccess ? GD_OK : GD_ERR_CUDA;
  };
  for (uint32_t i = 0; i < a->n_tensors; ++i) {
    const gd_adamw_tensor& t = a->tensors[i];
    if (t.n == 0) continue;
    const uint64_t need = (t.n + kChunk - 1) / kChunk;
    if (s.n_tensors == kMaxTensors || chunks + need > 0x7FFFFFFFull) {
      const int rc = flush();
      if (rc != GD_OK) return rc;
    }
    TensorEntry& e = table.t[s.n_tensors++];
    e.param = t.param;
    e.grad = t.grad;
    e.m = t.m;
    e.v = t.v;
    e.m_scale = t.m_scale;
    e.v_scale = t.v_scale;
    e.copy = t.copy;
    e.n = t.n;
    e.chunk0 = (uint32_t)chunks;
    e.index = i;
    e.decay = (float)(1.0 - a->lr * t.weight_decay);
    e.vectors = aligned_to(t.param, 4 * pb) && aligned_to(t.grad, 4 * gb) && aligned_to(t.m, 4 * sb) && aligned_to(t.v, 4 * sb) &&
                aligned_to(t.copy, 4 * cb);
    chunks += need;
  }
  return flush();
}
