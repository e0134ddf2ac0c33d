// One AdamW update of many tensors (gd_adamw_step): a stream over parameters, gradients and moments.
//
// The update is elementwise, so the bytes bound it: 28 per element with fp32 throughout, 16.1 with the moments in
// 8 bits - where the instructions (division and root to the last bit, random rounding, some 90 per element) come first.  One launch
// takes up to kMaxTensors tensors, whose table travels as the kernel argument (no device copy, no allocation); a CTA takes one
// chunk of kChunk consecutive elements of one tensor.  A warp works on blocks of 128 elements, four per lane in one 16-byte
// access, because 128 is also the unit that shares a scale in the 8-bit moments: its largest magnitude is one warp
// reduction, and nothing but the warp has to agree on it.  With 32-bit moments the next block waits in registers; with 8-bit ones,
// whose arithmetic needs them, three blocks are on their way into shared memory.
// A tensor whose buffers do not all start on a vector boundary (pieces of a flat vector do not), and a tensor's last,
// partial block, go element by element, lane-contiguous, with the same arithmetic.
//
// Measured (one B200): 138 M elements, 32 bits 575 us = 6.7 TB/s; 8 bits with bf16 gradients and copy 446 - 477 us by the clocks under sustained load
// (425 in short runs; 706 with the loads through registers and codes made one by one), 90 % of the issue slots used.
#include <cmath>

#include "gd_train.cuh"

namespace gd {
namespace {

constexpr uint32_t kAdamThreads = 256, kStride = kAdamThreads / 32 * 128;
template <int BITS>
constexpr uint32_t kChunk = (BITS == 8 ? 8 : 2) * kStride;   // elements a CTA takes: blocks a warp works through x its warps' stride

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

// Kernel arguments hold at most 32764 bytes.  The shorter tables are there because a launch pays for its argument's bytes.
constexpr uint32_t kFewTensors = 24, kSomeTensors = 110, kMaxTensors = 400;
template <uint32_t CAP>
struct AdamTable {
  AdamScalars s;
  TensorEntry t[CAP];
};
static_assert(sizeof(AdamTable<kMaxTensors>) <= 32764, "a kernel argument");

template <int DT>
__device__ __forceinline__ void load4(const void* base, uint32_t at, float (&x)[4]) {
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
__device__ __forceinline__ void store4(void* base, uint32_t at, const float (&x)[4]) {
  if constexpr (DT == GD_DTYPE_FP32)
    __stcs(reinterpret_cast<float4*>(static_cast<float*>(base) + at), make_float4(x[0], x[1], x[2], x[3]));
  else
    __stcs(reinterpret_cast<uint2*>(static_cast<uint16_t*>(base) + at), make_uint2(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3])));
}
template <int DT>
__device__ __forceinline__ float load1(const void* base, uint32_t at) {
  return Elem<DT>::get(static_cast<const typename Elem<DT>::type*>(base)[at]);
}
template <int DT>
__device__ __forceinline__ void store1(void* base, uint32_t at, float x) {
  static_cast<typename Elem<DT>::type*>(base)[at] = Elem<DT>::put(x);
}

__device__ __forceinline__ uint32_t mix32(uint32_t x) {
  x ^= x >> 16;
  x *= 0x7FEB352Du;
  x ^= x >> 15;
  x *= 0x846CA68Bu;
  return x ^ (x >> 16);
}

// fp8 (e4m3) of a magnitude y < 256, rounded up or down by 16 random bits.  In units of 2^-20 of the last bit kept a normal number
// is its own bits (exponent and mantissa run on); below 2^-6 the step is fixed, and y / 2 + 2^-7 has the bits that continue the
// normal numbers' downwards - it is also the larger of the two exactly there, so one maximum picks the case.  The code's seven bits
// come out in the top byte, 0xC0 too high; four of them are put right together by pack_codes().
// `low` is y / 2 + 2^-7.
__device__ __forceinline__ uint32_t encode_fp8(float y, float low, uint32_t random_bits_8_to_23) {
  return (__float_as_uint(fmaxf(y, low)) << 4) + random_bits_8_to_23;
}
// (top byte - 0xC0) of each: a code is below 0x80, so that is the sixth bit turned over and the seventh cleared
__device__ __forceinline__ uint32_t top_bytes(const uint32_t (&x)[4]) {
  return __byte_perm(__byte_perm(x[0], x[1], 0x0073), __byte_perm(x[2], x[3], 0x0073), 0x5410);
}
__device__ __forceinline__ uint32_t pack_codes(const uint32_t (&x)[4]) { return (top_bytes(x) ^ 0x40404040u) & 0x7F7F7F7Fu; }
// what is not finite becomes NaN
__device__ __forceinline__ uint32_t nan_codes(uint32_t codes, const float (&x)[4]) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (!(fabsf(x[j]) < INFINITY)) codes |= 0x7Fu << (8 * j);
  return codes;
}
__device__ __forceinline__ float2 decode_fp8x2(uint32_t two) {
  uint32_t h;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t)two));
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}

// The largest magnitude of a warp's values (NaN if there is one).
__device__ __forceinline__ float largest(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(fabsf(a)), "f"(fabsf(b)));
  return r;
}
__device__ __forceinline__ float warp_largest(float x) {
  float r;
  asm volatile("redux.sync.max.abs.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(x));
  return r;
}
// The same without what is not finite: an element that is held as NaN must not take the scale with it, which the other 127 need.
__device__ __forceinline__ float largest_finite(const float* x) {
  float top = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(x[j]) < INFINITY ? fabsf(x[j]) : 0.f);
  return warp_largest(top);
}
// The scale of a block from its largest magnitude, and its reciprocal: powers of two, so both products are exact.
__device__ __forceinline__ void block_scale(float top, float* scale, float* inverse) {
  const int e = max((int)(__float_as_uint(top) >> 23) - 7, 1);
  *scale = __uint_as_float((uint32_t)e << 23);
  *inverse = __uint_as_float((uint32_t)(254 - e) << 23);
}

// The update of two elements, in the order the header states: sums in pairs, the products that go into them singly, so that nothing is
// contracted.
__device__ __forceinline__ float2 apart(float2 a, float b) { return make_float2(__fmul_rn(a.x, b), __fmul_rn(a.y, b)); }
__device__ __forceinline__ void update(float* p, const float* grad, float* m, float* v, float* root, const AdamScalars& s, float scale, float decay) {
  const float2 g = mul2(make_float2(grad[0], grad[1]), both(scale)), c = mul2(g, both(s.one_minus_beta2));
  const float2 m2 = add2(apart(make_float2(m[0], m[1]), s.beta1), apart(g, s.one_minus_beta1));
  const float2 v2 = add2(apart(make_float2(v[0], v[1]), s.beta2), make_float2(__fmul_rn(c.x, g.x), __fmul_rn(c.y, g.y)));
  const float2 r = make_float2(__fsqrt_rn(v2.x), __fsqrt_rn(v2.y));
  const float2 d = add2(apart(r, s.root_factor), both(s.eps));
  const float2 q = apart(make_float2(__fdiv_rn(m2.x, d.x), __fdiv_rn(m2.y, d.y)), -s.step_size);
  const float2 p2 = add2(apart(make_float2(p[0], p[1]), decay), q);
  p[0] = p2.x, p[1] = p2.y;
  m[0] = m2.x, m[1] = m2.y;
  v[0] = v2.x, v[1] = v2.y;
  root[0] = r.x, root[1] = r.y;
}

// What a lane holds of a block: four elements.
template <int BITS>
struct Block {
  float p[4], g[4], m[4], v[4];
  uint32_t mc, vc;              // the 8-bit moments as they lie in memory, and their scales
  float ms, vs;
};

// The chunk of a CTA: the tensor's pointers moved to its start, so that everything in it is a 32-bit offset from an address the whole CTA shares.
struct Chunk {
  void* param;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  uint32_t n;
};
template <int PT, int GT>
__device__ __forceinline__ void load_block(Block<32>& b, const Chunk& t, uint32_t at, uint32_t lane) {
  load4<PT>(t.param, at + 4 * lane, b.p);
  load4<GT>(t.grad, at + 4 * lane, b.g);
  load4<GD_DTYPE_FP32>(t.m, at + 4 * lane, b.m);
  load4<GD_DTYPE_FP32>(t.v, at + 4 * lane, b.v);
}
// A block on its way through shared memory: parameters, gradients, codes of m and of v, the two scales.
constexpr int kStages = 4;
constexpr uint32_t kStageBytes = 512 + 512 + 128 + 128 + 16;
template <uint32_t BYTES>
__device__ __forceinline__ void ask(void* dst, const void* src) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(smem_u32(dst)), "l"(src), "n"(BYTES) : "memory");
}
template <int PT, int GT>
__device__ __forceinline__ void ask_block(unsigned char* stage, const Chunk& t, uint32_t at, uint32_t lane) {
  constexpr uint32_t pb = PT == GD_DTYPE_FP32 ? 16 : 8, gb = GT == GD_DTYPE_FP32 ? 16 : 8;
  const uint32_t e = at / 4 + lane;
  ask<pb>(stage + pb * lane, static_cast<const unsigned char*>(t.param) + e * pb);
  ask<gb>(stage + 512 + gb * lane, static_cast<const unsigned char*>(t.grad) + e * gb);
  ask<4>(stage + 1024 + 4 * lane, static_cast<const unsigned char*>(t.m) + e * 4);
  ask<4>(stage + 1152 + 4 * lane, static_cast<const unsigned char*>(t.v) + e * 4);
  if (lane < 2) ask<4>(stage + 1280 + 4 * lane, (lane ? t.v_scale : t.m_scale) + (at >> 7));
}
template <int DT>
__device__ __forceinline__ void take4(const unsigned char* p, uint32_t lane, float (&x)[4]) {
  if constexpr (DT == GD_DTYPE_FP32) {
    const float4 q = reinterpret_cast<const float4*>(p)[lane];
    x[0] = q.x, x[1] = q.y, x[2] = q.z, x[3] = q.w;
  } else {
    const uint2 q = reinterpret_cast<const uint2*>(p)[lane];
    const float2 a = unpack2<DT>(q.x), b = unpack2<DT>(q.y);
    x[0] = a.x, x[1] = a.y, x[2] = b.x, x[3] = b.y;
  }
}
template <int PT, int GT>
__device__ __forceinline__ void take_block(Block<8>& b, const unsigned char* stage, uint32_t lane) {
  take4<PT>(stage, lane, b.p);
  take4<GT>(stage + 512, lane, b.g);
  b.mc = reinterpret_cast<const uint32_t*>(stage + 1024)[lane];
  b.vc = reinterpret_cast<const uint32_t*>(stage + 1152)[lane];
  b.ms = reinterpret_cast<const float*>(stage + 1280)[0];
  b.vs = reinterpret_cast<const float*>(stage + 1280)[1];
}
// Element by element: element j of a lane is at + lane + 32 j.  What lies past the end is held as zeros.
template <int PT, int GT, int BITS>
__device__ __forceinline__ void load_ragged(Block<BITS>& b, const Chunk& t, uint32_t at, uint32_t lane) {
  b.mc = b.vc = 0u;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t e = at + lane + 32 * j;
    const bool in = e < t.n;
    b.p[j] = in ? load1<PT>(t.param, e) : 0.f;
    b.g[j] = in ? load1<GT>(t.grad, e) : 0.f;
    if constexpr (BITS == 32) {
      b.m[j] = in ? static_cast<const float*>(t.m)[e] : 0.f;
      b.v[j] = in ? static_cast<const float*>(t.v)[e] : 0.f;
    } else if (in) {
      b.mc |= (uint32_t)static_cast<const uint8_t*>(t.m)[e] << (8 * j);
      b.vc |= (uint32_t)static_cast<const uint8_t*>(t.v)[e] << (8 * j);
    }
  }
  if constexpr (BITS == 8) {
    b.ms = t.m_scale[at >> 7];
    b.vs = t.v_scale[at >> 7];
  }
}

// The update of a block; with 8-bit moments also their new codes (mc, vc) and scales (ms, vs).
template <bool RAGGED, int BITS>
__device__ __forceinline__ void update_block(Block<BITS>& b, const AdamScalars& s, float scale, float decay, uint32_t random_base, uint32_t first, uint32_t at,
                                             uint32_t n, uint32_t lane) {
  float root[4];
  if constexpr (BITS == 8) {
    const float2 m01 = decode_fp8x2(b.mc & 0xFFFFu), m23 = decode_fp8x2(b.mc >> 16);
    const float2 v01 = decode_fp8x2(b.vc & 0xFFFFu), v23 = decode_fp8x2(b.vc >> 16);
    const float2 ma = mul2(m01, both(b.ms)), mb = mul2(m23, both(b.ms)), ra = mul2(v01, both(b.vs)), rb = mul2(v23, both(b.vs));
    const float2 va = mul2(ra, ra), vb = mul2(rb, rb);
    b.m[0] = ma.x, b.m[1] = ma.y, b.m[2] = mb.x, b.m[3] = mb.y;
    b.v[0] = va.x, b.v[1] = va.y, b.v[2] = vb.x, b.v[3] = vb.y;
  }
#pragma unroll
  for (int j = 0; j < 4; j += 2) update(b.p + j, b.g + j, b.m + j, b.v + j, root + j, s, scale, decay);
  if constexpr (BITS == 8) {
    if constexpr (RAGGED) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (at + lane + 32 * j >= n) b.m[j] = root[j] = 0.f;
    }
    float m_top = warp_largest(largest(largest(b.m[0], b.m[1]), largest(b.m[2], b.m[3])));
    float v_top = warp_largest(largest(largest(root[0], root[1]), largest(root[2], root[3])));
    const bool finite = m_top < INFINITY && v_top < INFINITY;      // the same for the whole warp
    if (!finite) m_top = largest_finite(b.m), v_top = largest_finite(root);
    float m_inverse, v_inverse;
    block_scale(m_top, &b.ms, &m_inverse);
    block_scale(v_top, &b.vs, &v_inverse);
    uint32_t cm[4], cv[4];
#pragma unroll
    for (int j = 0; j < 4; j += 2) {
      const float2 ym = mul2(make_float2(fabsf(b.m[j]), fabsf(b.m[j + 1])), both(m_inverse));
      float2 yv = mul2(make_float2(root[j], root[j + 1]), both(v_inverse));
      if (root[j] > 0.f) yv.x = fmaxf(yv.x, 0x1p-9f);        // at least the smallest positive code, whose step this is
      if (root[j + 1] > 0.f) yv.y = fmaxf(yv.y, 0x1p-9f);
      const float2 lm = fma2(ym, both(0.5f), both(0x1p-7f)), lv = fma2(yv, both(0.5f), both(0x1p-7f));
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t e = first + at + (RAGGED ? lane + 32 * (j + i) : 4 * lane + j + i);
        const uint32_t h = mix32(e * 0x9E3779B9u + random_base);
        cm[j + i] = encode_fp8(i ? ym.y : ym.x, i ? lm.y : lm.x, __byte_perm(h, 0u, 0x4324));
        cv[j + i] = encode_fp8(i ? yv.y : yv.x, i ? lv.y : lv.x, __byte_perm(h, 0u, 0x4104));
      }
    }
    const uint32_t signs[4] = {__float_as_uint(b.m[0]), __float_as_uint(b.m[1]), __float_as_uint(b.m[2]), __float_as_uint(b.m[3])};
    b.mc = pack_codes(cm);
    b.vc = pack_codes(cv);
    if (!finite) {
      b.mc = nan_codes(b.mc, b.m);
      b.vc = nan_codes(b.vc, root);
    }
    b.mc |= top_bytes(signs) & 0x80808080u;
  }
}

template <int PT, int BITS>
__device__ __forceinline__ void store_block(const Block<BITS>& b, const Chunk& t, int copy_dtype, uint32_t at, uint32_t lane) {
  store4<PT>(t.param, at + 4 * lane, b.p);
  if (t.copy) {
    if (copy_dtype == GD_DTYPE_BF16) store4<GD_DTYPE_BF16>(t.copy, at + 4 * lane, b.p);
    else if (copy_dtype == GD_DTYPE_FP16) store4<GD_DTYPE_FP16>(t.copy, at + 4 * lane, b.p);
    else store4<GD_DTYPE_FP32>(t.copy, at + 4 * lane, b.p);
  }
  if constexpr (BITS == 32) {
    store4<GD_DTYPE_FP32>(t.m, at + 4 * lane, b.m);
    store4<GD_DTYPE_FP32>(t.v, at + 4 * lane, b.v);
  } else {
    __stcs(reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.m) + at + 4 * lane), b.mc);
    __stcs(reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(t.v) + at + 4 * lane), b.vc);
  }
}
template <int PT, int BITS>
__device__ __forceinline__ void store_ragged(const Block<BITS>& b, const Chunk& t, int copy_dtype, uint32_t at, uint32_t lane) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const uint32_t e = at + lane + 32 * j;
    if (e >= t.n) continue;
    store1<PT>(t.param, e, b.p[j]);
    if (t.copy) {
      if (copy_dtype == GD_DTYPE_BF16) store1<GD_DTYPE_BF16>(t.copy, e, b.p[j]);
      else if (copy_dtype == GD_DTYPE_FP16) store1<GD_DTYPE_FP16>(t.copy, e, b.p[j]);
      else store1<GD_DTYPE_FP32>(t.copy, e, b.p[j]);
    }
    if constexpr (BITS == 32) {
      static_cast<float*>(t.m)[e] = b.m[j];
      static_cast<float*>(t.v)[e] = b.v[j];
    } else {
      static_cast<uint8_t*>(t.m)[e] = (uint8_t)(b.mc >> (8 * j));
      static_cast<uint8_t*>(t.v)[e] = (uint8_t)(b.vc >> (8 * j));
    }
  }
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
  const TensorEntry& of = table.t[lo];
  const uint64_t start = (uint64_t)(blockIdx.x - of.chunk0) * kChunk<BITS>;
  const uint32_t end = (uint32_t)min(of.n - start, (uint64_t)kChunk<BITS>), first = (uint32_t)start;
  const uint32_t pb = sizeof(typename Elem<PT>::type), gb = sizeof(typename Elem<GT>::type), cb = s.copy_dtype == GD_DTYPE_FP32 ? 4 : 2, sb = BITS / 8;
  Chunk t;
  t.param = static_cast<char*>(of.param) + start * pb;
  t.grad = static_cast<const char*>(of.grad) + start * gb;
  t.m = static_cast<char*>(of.m) + start * sb;
  t.v = static_cast<char*>(of.v) + start * sb;
  t.copy = of.copy ? static_cast<char*>(of.copy) + start * cb : nullptr;
  t.m_scale = of.m_scale + start / 128;
  t.v_scale = of.v_scale + start / 128;
  t.n = end;
  const float decay = of.decay;
  const bool vectors = of.vectors;
  const uint32_t lane = lane_id(), random_base = s.seed + of.index * 0x85EBCA77u;
  uint32_t at = (threadIdx.x >> 5) * 128u;
  pdl_wait();
  pdl_trigger();
  const float scale = s.grad_scale_dev ? __fmul_rn(s.grad_scale, *s.grad_scale_dev) : s.grad_scale;
  Block<BITS> b;
  if constexpr (BITS == 8) {
    extern __shared__ __align__(16) unsigned char smem[];
    if (vectors && at + 128u <= end) {
      unsigned char* ring = smem + (threadIdx.x >> 5) * (kStages * kStageBytes);
      uint32_t ask = at;
#pragma unroll
      for (int i = 0; i < kStages - 1; ++i, ask += kStride) {
        if (ask + 128u <= end) ask_block<PT, GT>(ring + i * kStageBytes, t, ask, lane);
        asm volatile("cp.async.commit_group;" ::: "memory");
      }
      for (uint32_t i = 0; at + 128u <= end; ++i, at += kStride, ask += kStride) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 2) : "memory");
        __syncwarp();                      // everybody's part of this block has landed, and the block before it has been read
        if (ask + 128u <= end) ask_block<PT, GT>(ring + (i + kStages - 1) % kStages * kStageBytes, t, ask, lane);
        asm volatile("cp.async.commit_group;" ::: "memory");
        take_block<PT, GT>(b, ring + i % kStages * kStageBytes, lane);
        update_block<false, BITS>(b, s, scale, decay, random_base, first, at, end, lane);
        if (lane == 0) t.m_scale[at >> 7] = b.ms, t.v_scale[at >> 7] = b.vs;
        store_block<PT, BITS>(b, t, s.copy_dtype, at, lane);
      }
    }
  } else {
    Block<BITS> next;
    if (vectors && at + 128u <= end) {
      load_block<PT, GT>(b, t, at, lane);
      while (true) {
        const uint32_t after = at + kStride;
        const bool more = after + 128u <= end;
        if (more) load_block<PT, GT>(next, t, after, lane);        // under way while this block is worked on
        update_block<false, BITS>(b, s, scale, decay, random_base, first, at, end, lane);
        store_block<PT, BITS>(b, t, s.copy_dtype, at, lane);
        at = after;
        if (!more) break;
        b = next;
      }
    }
  }
  if (at < end) load_ragged<PT, GT, BITS>(b, t, at, lane);
  while (at < end) {
    Block<BITS> next;
    if (at + kStride < end) load_ragged<PT, GT, BITS>(next, t, at + kStride, lane);
    update_block<true, BITS>(b, s, scale, decay, random_base, first, at, end, lane);
    if constexpr (BITS == 8) {
      if (lane == 0) t.m_scale[at >> 7] = b.ms, t.v_scale[at >> 7] = b.vs;
    }
    store_ragged<PT, BITS>(b, t, s.copy_dtype, at, lane);
    b = next;
    at += kStride;
  }
}

template <int PT, int GT, int BITS>
cudaError_t launch_cap(const AdamTable<kMaxTensors>& full, uint32_t chunks, cudaStream_t stream) {
  constexpr size_t smem = BITS == 8 ? kAdamThreads / 32 * kStages * kStageBytes : 0;
  static_assert(smem <= 48 * 1024, "without asking for more shared memory");
  const auto with = [&](auto& table) {
    table.s = full.s;
    for (uint32_t i = 0; i < full.s.n_tensors; ++i) table.t[i] = full.t[i];
  };
  if (full.s.n_tensors <= kFewTensors) {
    AdamTable<kFewTensors> few;
    with(few);
    return launch_dependent(adamw_kernel<PT, GT, BITS, kFewTensors>, dim3(chunks), dim3(kAdamThreads), smem, stream, few);
  }
  if (full.s.n_tensors <= kSomeTensors) {
    AdamTable<kSomeTensors> some;
    with(some);
    return launch_dependent(adamw_kernel<PT, GT, BITS, kSomeTensors>, dim3(chunks), dim3(kAdamThreads), smem, stream, some);
  }
  return launch_dependent(adamw_kernel<PT, GT, BITS, kMaxTensors>, dim3(chunks), dim3(kAdamThreads), smem, stream, full);
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
  const uint64_t chunk = eight ? kChunk<8> : kChunk<32>;
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
    const uint64_t need = (t.n + chunk - 1) / chunk;
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
