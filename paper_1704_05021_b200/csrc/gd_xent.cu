// Softmax cross-entropy of a batch and the gradient of its logits (gd_cross_entropy).
//
// Every logit is read from memory once and every gradient written once; between the two the row waits on the chip, so the
// bytes bound it (2 x 2 B per logit in 16 bits), and in 16 bits the two exponentials per logit come close behind: they alone would take
// 70 % of that time.  Long rows: a cluster of 1 .. 8 CTAs takes one row, each a slice of it, which bulk copies bring into
// shared memory (what a slice has beyond that is read a second time, from L2).  While it arrives each thread keeps a running
// maximum and the sum of exp(x - maximum) of what it has seen; the pairs are joined over warps, the CTA and - sent into the
// others' shared memory and counted there, which spares the fence that a cluster barrier puts behind every access - the cluster, always
// in the same order.  Then the gradient goes out from shared memory.  Short rows (up to kShortClasses classes): a group of 4 .. 32
// lanes holds a row in registers.  exp(x - m) subtracts first, in fp32: the difference is exact where it matters, and masked or
// lowest-value logits give 0 and never a NaN.
//
// Measured (one B200): 4000 x 85000 in bf16 266 us = 5.1 TB/s under sustained load, 246 in short runs (361 by plain loads,
// two passes over shared memory and cluster barriers); 1.0 GB of fp32 rows of 2048 .. 85000 6.3 - 6.7 TB/s.
#include <algorithm>
#include <type_traits>

#include "gd_mma.cuh"

namespace gd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -INFINITY;
// Most 16-byte pieces of a slice for 32, 64 and 128 threads.  Measured on 85 M logits (us, 32 / 64 / 128 / 256 threads): rows of 2048 in
// bf16 66 / 84 / 119 / 226, of 8192 72 / 60 / 65 / 92, of 85000 127 / 87 / 70 / 74, of 200000 in fp32 398 / 228 / 157 / 132.
constexpr uint32_t kVecs32 = 256, kVecs64 = 1024, kVecs128 = 3584;
constexpr uint32_t kShortClasses = 1024;       // 32 lanes x 32 registers
constexpr uint32_t kSliceBytes = 48u << 10;    // a slice this long leaves room for four CTAs on an SM: one's loads run under another's sums and stores
constexpr uint32_t kParts = 4;                 // bulk copies a slice arrives by: the maximum is taken of one while the others are under way
constexpr uint32_t kMaxStage = 200u << 10;     // shared memory a CTA may ask for its slice

struct XentArgs {
  const void* logits;
  void* grad;
  const void* targets;
  uint64_t ld_logits, ld_grad, rows;
  uint32_t classes, target_bits;
  int64_t ignore_index;
  float grad_scale;
  const float* grad_scale_dev;
  float* loss;
  float* lse;
};

// exp(d) for d <= 0; below 2^-126 it is 0
__device__ __forceinline__ float exp_of(float d) {
  float e;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(d * kLog2e));
  return e;
}
// the target of a row: >= 0 a class, -1 none (ignored), -2 out of range
__device__ __forceinline__ int64_t target_of(const XentArgs& a, uint64_t row) {
  const int64_t t = a.target_bits == 64 ? static_cast<const int64_t*>(a.targets)[row] : static_cast<const int32_t*>(a.targets)[row];
  if (t == a.ignore_index) return -1;
  return t >= 0 && t < (int64_t)a.classes ? t : -2;
}
// (m, s) <- the join of (m, s) and (om, os).  A side of masked classes has m = -inf and s = 0, or the NaN that was among them.
__device__ __forceinline__ void join(float& m, float& s, float om, float os) {
  const float top = fmaxf(m, om);
  const float a = m == kNegInf ? s : s * exp_of(m - top);
  const float b = om == kNegInf ? os : os * exp_of(om - top);
  m = top;
  s = a + b;
}

// What a row's statistics say: log-sum-exp, loss, and the two numbers the gradient takes: exp(x - m) * factor - (j == t) * scale.
struct RowResult {
  float lse, loss, factor, scale;
};
__device__ __forceinline__ RowResult finish(float m, float s, int64_t t, float target_logit, float scale) {
  RowResult r;
  const float log_s = logf(s);
  r.lse = s == 0.f ? m : m + log_s;              // (every class masked: -inf)
  r.scale = scale;
  r.factor = scale / s;
  r.loss = (m - target_logit) + log_s;
  if (t == -1) r.loss = 0.f, r.scale = 0.f, r.factor = 0.f;
  if (t == -2 || (t >= 0 && s == 0.f)) r.loss = r.factor = r.scale = NAN;
  return r;
}

template <int DT>
struct Vec {   // 16 bytes of logits
  static constexpr uint32_t kElems = DT == GD_DTYPE_FP32 ? 4 : 8;
  static __device__ __forceinline__ void get(const uint4& q, float (&x)[kElems]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (DT == GD_DTYPE_FP32) {
        x[i] = __uint_as_float(w[i]);
      } else {
        const float2 f = unpack2<DT>(w[i]);
        x[2 * i] = f.x, x[2 * i + 1] = f.y;
      }
    }
  }
  static __device__ __forceinline__ uint4 put(const float (&x)[kElems]) {
    if constexpr (DT == GD_DTYPE_FP32)
      return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
    else
      return make_uint4(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]), pack2<DT>(x[4], x[5]), pack2<DT>(x[6], x[7]));
  }
};

// The largest of a piece (two at a time as they lie, in 16 bits: nothing to round), and the sum of exp(x - base), as trees: the
// loops around them are bound by latency otherwise.
template <int DT>
__device__ __forceinline__ float top_of(const uint4& q) {
  if constexpr (DT == GD_DTYPE_FP32) {
    return fmaxf(fmaxf(__uint_as_float(q.x), __uint_as_float(q.y)), fmaxf(__uint_as_float(q.z), __uint_as_float(q.w)));
  } else {
    using T2 = typename std::conditional<DT == GD_DTYPE_BF16, __nv_bfloat162, __half2>::type;
    const auto as = [](uint32_t w) { return *reinterpret_cast<const T2*>(&w); };
    const T2 m = __hmax2(__hmax2(as(q.x), as(q.y)), __hmax2(as(q.z), as(q.w)));
    const float2 f = unpack2<DT>(*reinterpret_cast<const uint32_t*>(&m));
    return fmaxf(f.x, f.y);
  }
}
// exp(x - base) of a piece, in pairs
template <int DT>
__device__ __forceinline__ void exps_of(const uint4& q, float base, float2 (&e)[Vec<DT>::kElems / 2]) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
  const float2 less = make_float2(-base, -base), log2e = make_float2(kLog2e, kLog2e);
#pragma unroll
  for (uint32_t j = 0; j < Vec<DT>::kElems / 2; ++j) {
    float2 f;
    if constexpr (DT == GD_DTYPE_FP32) f = make_float2(__uint_as_float(w[2 * j]), __uint_as_float(w[2 * j + 1]));
    else f = unpack2<DT>(w[j]);
    f = mul2(add2(f, less), log2e);
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e[j].x) : "f"(f.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e[j].y) : "f"(f.y));
  }
}
template <int DT>
__device__ __forceinline__ float sum_of(const uint4& q, float base) {
  constexpr uint32_t P = Vec<DT>::kElems / 2;
  float2 e[P];
  exps_of<DT>(q, base, e);
#pragma unroll
  for (uint32_t w = P / 2; w > 0; w >>= 1) {
#pragma unroll
    for (uint32_t j = 0; j < w; ++j) e[j] = add2(e[j], e[j + w]);
  }
  return e[0].x + e[0].y;
}
// The gradient of a piece whose first class is e0: exp(x - m) * factor, less `scale` at the target.
template <int DT>
__device__ __forceinline__ uint4 gradient_of(const uint4& q, float m, const RowResult& r, bool none, uint32_t e0, uint32_t hit) {
  constexpr uint32_t V = Vec<DT>::kElems;
  if (none) return make_uint4(0u, 0u, 0u, 0u);
  float2 e[V / 2];
  exps_of<DT>(q, m, e);
  float f[V];
#pragma unroll
  for (uint32_t j = 0; j < V / 2; ++j) {
    e[j] = mul2(e[j], make_float2(r.factor, r.factor));
    f[2 * j] = e[j].x, f[2 * j + 1] = e[j].y;
  }
  if (hit - e0 < V) {
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) f[j] -= e0 + j == hit ? r.scale : 0.f;
  }
  return Vec<DT>::put(f);
}

// One row per cluster.  `slice`: elements per CTA (a multiple of 64), `stage`: how many of them shared memory holds (a multiple of 8).
// Where the row's first address and the gradient's agree modulo 16 bytes the slice is worked on in 16-byte pieces, its ragged
// ends element by element; otherwise all of it element by element.
template <int DT, uint32_t THREADS>
__global__ void __launch_bounds__(THREADS) xent_row_kernel(const __grid_constant__ XentArgs a, uint32_t cluster, uint32_t slice, uint32_t stage) {
  using T = typename Elem<DT>::type;
  constexpr uint32_t V = Vec<DT>::kElems;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float2 s_warp[THREADS / 32];
  __shared__ __align__(8) float2 s_pairs[8];
  __shared__ uint64_t s_full[kParts], s_pairs_in;
  __shared__ float s_target;
  const uint32_t tid = threadIdx.x, rank = cluster > 1 ? cluster_rank() : 0u;
  const uint64_t row = blockIdx.x / cluster;
  const uint32_t c0 = min(rank * slice, a.classes), c1 = min(c0 + slice, a.classes), len = c1 - c0;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld_logits + c0;
  T* out = a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad + c0 : nullptr;
  if (tid == 0) {
    for (uint32_t p = 0; p < kParts; ++p) mbar_init(&s_full[p], 1u);
    mbar_init(&s_pairs_in, 1u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    mbar_arrive_expect_tx(&s_pairs_in, cluster * 8u);
  }
  __syncthreads();
  if (cluster > 1) cluster_arrive_relaxed();
  pdl_wait();
  pdl_trigger();
  // [0, head) and [body, len) element by element, [head, body) in pieces of 16 bytes whose addresses are multiples of 16
  const bool pieces = !out || ((uintptr_t)out & 15u) == ((uintptr_t)x & 15u);
  const uint32_t head = pieces ? min((V - (uint32_t)((uintptr_t)x & 15u) / (uint32_t)sizeof(T)) % V, len) : 0u;
  const uint32_t n_vec = pieces ? (len - head) / V : 0u, body = pieces ? head + n_vec * V : 0u;
  const uint32_t rest = pieces ? head + (len - body) : len;       // elements outside the pieces: read from memory each time
  // shared memory holds the first `kept` pieces (all of them, usually), brought by bulk copies in kParts parts
  const uint32_t kept = min(n_vec, stage / V), part = ((kept + kParts - 1) / kParts + 7u) & ~7u;
  const uint4* held_vec = reinterpret_cast<const uint4*>(smem);
  const uint4* x_vec = reinterpret_cast<const uint4*>(x + head);
  if (tid == 0) {
    for (uint32_t p = 0; p < kParts; ++p) {
      const uint32_t v0 = min(p * part, kept), v1 = min(v0 + part, kept);
      mbar_arrive_expect_tx(&s_full[p], (v1 - v0) * 16u);
      if (v1 > v0) bulk_load(smem + v0 * 16u, x_vec + v0, (v1 - v0) * 16u, &s_full[p]);
    }
  }
  const int64_t target = target_of(a, row);
  const float scale = a.grad_scale_dev ? a.grad_scale * *a.grad_scale_dev : a.grad_scale;
  const bool answers = tid == 0 && rank == 0;      // writes the row's loss, and so reads the target's logit, wherever it lies
  const float target_logit = answers && target >= 0 ? Elem<DT>::get(static_cast<const T*>(a.logits)[row * a.ld_logits + target]) : 0.f;
  bool landed = true;

  // Each thread's running maximum and sum: the sum is rescaled when a piece raises the maximum.
  float m = kNegInf, s = 0.f;                    // (a NaN is passed over by the maximum and turns up in the sum)
  const auto take = [&](const uint4& q) {
    const float top = fmaxf(m, top_of<DT>(q)), base = top == kNegInf ? 0.f : top;     // (masked classes only so far: exp(-inf) = 0, or the NaN among them)
    s = s * exp_of(m - base) + sum_of<DT>(q, base);
    m = top;
  };
  for (uint32_t e = tid; e < rest; e += THREADS) {
    const float f = Elem<DT>::get(x[e < head ? e : body + (e - head)]), top = fmaxf(m, f), base = top == kNegInf ? 0.f : top;
    s = s * exp_of(m - base) + exp_of(f - base);
    m = top;
  }
  for (uint32_t i = kept + tid; i < n_vec; i += THREADS) take(__ldcg(x_vec + i));
  const int never = 0;
  for (uint32_t p = 0; p < kParts; ++p) {
    landed = mbar_wait(&s_full[p], 0u, &never) && landed;       // (also behind a wait that ran out: the CTA must not end with copies under way)
    const uint32_t v1 = min((p + 1) * part, kept);
    for (uint32_t i = p * part + tid; i < v1; i += THREADS) take(held_vec[i]);
  }
  if (!landed) s = NAN;                          // (a copy that never came: the row's results say so)
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) join(m, s, __shfl_xor_sync(0xFFFFFFFFu, m, o), __shfl_xor_sync(0xFFFFFFFFu, s, o));
  if ((tid & 31u) == 0u) s_warp[tid >> 5] = make_float2(m, s);
  // In place, the target's logit is overwritten by whichever CTA has it in its slice, once that has this one's pair: the read is over
  // before the pair is sent (its value goes through shared memory ahead of the barrier), not merely begun.
  if (answers) s_target = target_logit;
  __syncthreads();
  m = s_warp[0].x, s = s_warp[0].y;
#pragma unroll
  for (uint32_t w = 1; w < THREADS / 32; ++w) join(m, s, s_warp[w].x, s_warp[w].y);
  if (cluster > 1) {
    // to every CTA of the cluster, counted there in bytes: no fence over this CTA's memory traffic, as a barrier would need
    cluster_wait();                              // (everybody's mbarrier exists: arrived at long ago)
    if (tid < cluster) send_peer2(peer_address(smem_u32(&s_pairs[rank]), tid), make_float2(m, s), peer_address(smem_u32(&s_pairs_in), tid));
    landed = mbar_wait(&s_pairs_in, 0u, &never);
    m = kNegInf, s = landed ? 0.f : NAN;
    for (uint32_t r = 0; r < cluster; ++r) join(m, s, s_pairs[r].x, s_pairs[r].y);
    cluster_arrive_relaxed();                    // the pairs have been received; waited for before this CTA ends
  }
  const RowResult r = finish(m, s, target, answers ? s_target : 0.f, scale);
  if (answers) {
    if (a.loss) a.loss[row] = r.loss;
    if (a.lse) a.lse[row] = r.lse;
  }
  if (out) {
    const uint32_t hit = target >= (int64_t)c0 && target < (int64_t)c1 ? (uint32_t)(target - c0) : 0xFFFFFFFFu;
    const bool none = target == -1;              // 0 whatever the logits: not 0 * NaN
    uint4* out_vec = reinterpret_cast<uint4*>(out + head);
#pragma unroll 2
    for (uint32_t i = tid; i < kept; i += THREADS) __stcs(out_vec + i, gradient_of<DT>(held_vec[i], m, r, none, head + i * V, hit));
    for (uint32_t i = kept + tid; i < n_vec; i += THREADS)      // the second read of these: from L2, usually
      __stcs(out_vec + i, gradient_of<DT>(__ldcg(x_vec + i), m, r, none, head + i * V, hit));
    for (uint32_t i = tid; i < rest; i += THREADS) {
      const uint32_t e = i < head ? i : body + (i - head);
      const float g = none ? 0.f : exp_of(Elem<DT>::get(x[e]) - m) * r.factor;
      out[e] = Elem<DT>::put(g - (e == hit ? r.scale : 0.f));
    }
  }
  if (cluster > 1) cluster_wait();
}

// Short rows: G lanes hold a row, PER elements each (element j of a lane is class lane + j G).
template <int DT, int G, int PER>
__global__ void __launch_bounds__(128) xent_short_kernel(const __grid_constant__ XentArgs a) {
  using T = typename Elem<DT>::type;
  const uint64_t row = ((uint64_t)blockIdx.x * 128u + threadIdx.x) / G;
  const uint32_t lane = threadIdx.x % G;
  pdl_wait();
  pdl_trigger();
  const bool live = row < a.rows;
  const int64_t target = live ? target_of(a, row) : -1;
  const float scale = a.grad_scale_dev ? a.grad_scale * *a.grad_scale_dev : a.grad_scale;
  const T* x = static_cast<const T*>(a.logits) + (live ? row : 0) * a.ld_logits;
  float f[PER], m = kNegInf;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const uint32_t c = lane + j * G;
    f[j] = live && c < a.classes ? Elem<DT>::get(x[c]) : kNegInf;
    m = fmaxf(m, f[j]);
  }
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  const float base = m == kNegInf ? 0.f : m;
  float s = 0.f, target_logit = 0.f;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    if ((int64_t)(lane + j * G) == target) target_logit = f[j];
    f[j] = exp_of(f[j] - base);
    s += f[j];
  }
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) {
    s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
    target_logit += __shfl_xor_sync(0xFFFFFFFFu, target_logit, o);      // (one lane holds it, the others 0)
  }
  if (!live) return;
  const RowResult r = finish(m, s, target, target_logit, scale);
  if (lane == 0) {
    if (a.loss) a.loss[row] = r.loss;
    if (a.lse) a.lse[row] = r.lse;
  }
  if (!a.grad) return;
  T* out = static_cast<T*>(a.grad) + row * a.ld_grad;
#pragma unroll
  for (int j = 0; j < PER; ++j) {
    const uint32_t c = lane + j * G;
    if (c < a.classes) out[c] = Elem<DT>::put(target == -1 ? 0.f : f[j] * r.factor - ((int64_t)c == target ? r.scale : 0.f));
  }
}

template <int DT, int G, int PER>
cudaError_t launch_short(const XentArgs& a, cudaStream_t stream) {
  const uint64_t blocks = (a.rows * G + 127) / 128;
  return launch_dependent(xent_short_kernel<DT, G, PER>, dim3((uint32_t)blocks), dim3(128), 0, stream, a);
}

template <int DT, uint32_t THREADS>
cudaError_t launch_clusters(const XentArgs& a, uint32_t cluster, uint32_t slice, uint32_t stage, cudaStream_t stream) {
  auto kernel = xent_row_kernel<DT, THREADS>;
  // Always: without it a CTA has 48 KB for its static and its dynamic shared memory together, and the slice alone may be that long.
  static PerDeviceInt ready;
  int dev;
  if (!ready.get(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxStage);
    if (e != cudaSuccess) return e;
    ready.set(dev, 1);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)(a.rows * cluster));
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = stage * sizeof(typename Elem<DT>::type);
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kernel, a, cluster, slice, stage);
}

template <int DT>
cudaError_t launch_rows(const XentArgs& a, cudaStream_t stream) {
  constexpr uint32_t item = DT == GD_DTYPE_FP32 ? 4 : 2;
  const uint32_t c = a.classes;
  if (c <= 16) return launch_short<DT, 4, 4>(a, stream);
  if (c <= 64) return launch_short<DT, 8, 8>(a, stream);
  if (c <= 256) return launch_short<DT, 32, 8>(a, stream);
  if (c <= kShortClasses) return launch_short<DT, 32, 32>(a, stream);
  // CTAs per row: enough that a slice leaves room for others on its SM; more while the rows alone do not fill the GPU
  // and a slice stays long enough to keep its threads busy
  uint32_t cluster = 1;
  while (cluster < 8 && ((uint64_t)c * item > (uint64_t)cluster * kSliceBytes ||
                         (a.rows * cluster * 2 <= (uint64_t)sm_count() && c / (2 * cluster) >= 2048)))
    cluster *= 2;
  const uint32_t slice = ((c + cluster - 1) / cluster + 63) / 64 * 64;
  const uint32_t stage = std::min(slice * item, kMaxStage) / item;
  // threads by what each has to do: a short slice would pay for more of them in synchronisation, not gain by them
  const uint32_t vecs = slice * item / 16;
  if (vecs <= kVecs32) return launch_clusters<DT, 32>(a, cluster, slice, stage, stream);
  if (vecs <= kVecs64) return launch_clusters<DT, 64>(a, cluster, slice, stage, stream);
  if (vecs <= kVecs128) return launch_clusters<DT, 128>(a, cluster, slice, stage, stream);
  return launch_clusters<DT, 256>(a, cluster, slice, stage, stream);
}

}  // namespace
}  // namespace gd

extern "C" int gd_cross_entropy(const gd_cross_entropy_args* g, void* stream_v) {
  using namespace gd;
  if (!g || g->reserved != 0 || !is_dtype(g->dtype) || (g->target_bits != 32 && g->target_bits != 64)) return GD_ERR_INVALID_ARG;
  if (g->classes == 0) return GD_ERR_INVALID_ARG;
  if (g->rows >> 31 || g->classes >> 31) return GD_ERR_TOO_LARGE;
  if (g->rows == 0) return GD_OK;
  const size_t item = dtype_bytes(g->dtype);
  if (!g->logits || !g->targets || (!g->loss && !g->lse && !g->grad)) return GD_ERR_INVALID_ARG;
  if (!aligned_to(g->logits, item) || !aligned_to(g->grad, item) || !aligned_to(g->targets, (size_t)g->target_bits / 8) || !aligned_to(g->loss, 4) ||
      !aligned_to(g->lse, 4) || !aligned_to(g->grad_scale_dev, 4))
    return GD_ERR_INVALID_ARG;
  if (g->rows > 1 && (g->ld_logits < g->classes || (g->grad && g->ld_grad < g->classes))) return GD_ERR_INVALID_ARG;
  if (g->grad == g->logits && g->rows > 1 && g->ld_grad != g->ld_logits) return GD_ERR_INVALID_ARG;
  XentArgs a;
  a.logits = g->logits;
  a.grad = g->grad;
  a.targets = g->targets;
  a.ld_logits = g->ld_logits;
  a.ld_grad = g->ld_grad;
  a.rows = g->rows;
  a.classes = (uint32_t)g->classes;
  a.target_bits = (uint32_t)g->target_bits;
  a.ignore_index = g->ignore_index;
  a.grad_scale = g->grad_scale;
  a.grad_scale_dev = g->grad_scale_dev;
  a.loss = g->loss;
  a.lse = g->lse;
  cudaStream_t stream = (cudaStream_t)stream_v;
  // a grid holds 2^31 - 1 CTAs: more rows than that many clusters go in several launches
  const uint64_t most = 0x7FFFFFFFull / 8;
  for (uint64_t at = 0; at < g->rows; at += most) {
    XentArgs b = a;
    b.rows = g->rows - at < most ? g->rows - at : most;
    b.logits = (const char*)a.logits + at * a.ld_logits * item;
    b.grad = a.grad ? (char*)a.grad + at * a.ld_grad * item : nullptr;
    b.targets = (const char*)a.targets + at * (uint64_t)(g->target_bits / 8);
    b.loss = a.loss ? a.loss + at : nullptr;
    b.lse = a.lse ? a.lse + at : nullptr;
    ProfileScope ps(stream, PT_XENT);
    cudaError_t e;
    switch (g->dtype) {
      case GD_DTYPE_FP32: e = launch_rows<GD_DTYPE_FP32>(b, stream); break;
      case GD_DTYPE_BF16: e = launch_rows<GD_DTYPE_BF16>(b, stream); break;
      default: e = launch_rows<GD_DTYPE_FP16>(b, stream); break;
    }
    if (e != cudaSuccess) return GD_ERR_CUDA;
    note_launches(1);
  }
  return GD_OK;
}
