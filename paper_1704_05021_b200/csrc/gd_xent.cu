// Softmax cross-entropy of a batch and the gradient of its logits (gd_cross_entropy).
//
// Every logit is read from memory once and every gradient written once; between the two the row waits on the chip, so the
// bytes bound it (2 x 2 B per logit in 16 bits).  Long rows: a cluster of 1 .. 8 CTAs takes one row, each a slice of it, which it
// keeps in shared memory as it arrives (what a slice has beyond that is read a second time).  A CTA finds the maximum m of its slice
// while loading and sum exp(x - m) from shared memory; the CTAs of a cluster exchange their (m, sum) pairs through distributed
// shared memory and each joins them in the same order.  Short rows (up to kShortClasses classes): a group of 4 .. 32 lanes holds a row in
// registers.  exp(x - m) subtracts first, in fp32: the difference is exact where it matters, and masked or lowest-value
// logits give 0 and never a NaN.
#include "gd_mma.cuh"

namespace gd {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kNegInf = -INFINITY;
constexpr uint32_t kRowThreads = 256;
constexpr uint32_t kShortClasses = 1024;       // 32 lanes x 32 registers
constexpr uint32_t kSliceBytes = 40u << 10;    // a slice this long leaves room for five CTAs on an SM: one's loads run under another's sums and stores
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

// One row per cluster.  `slice`: elements per CTA (a multiple of 64), `stage`: how many of them shared memory holds (a multiple of 8).
// Where the row's first address and the gradient's agree modulo 16 bytes the slice is worked on in 16-byte pieces, its ragged
// ends element by element; otherwise all of it element by element.
template <int DT>
__global__ void __launch_bounds__(kRowThreads) xent_row_kernel(const __grid_constant__ XentArgs a, uint32_t cluster, uint32_t slice, uint32_t stage) {
  using T = typename Elem<DT>::type;
  constexpr uint32_t V = Vec<DT>::kElems;
  extern __shared__ __align__(16) unsigned char smem[];
  __shared__ float s_warp[kRowThreads / 32][2];
  __shared__ float2 s_pair;
  __shared__ uint64_t s_full[kParts];
  const uint32_t tid = threadIdx.x, rank = cluster > 1 ? cluster_rank() : 0u;
  const uint64_t row = blockIdx.x / cluster;
  const uint32_t c0 = min(rank * slice, a.classes), c1 = min(c0 + slice, a.classes), len = c1 - c0;
  const T* x = static_cast<const T*>(a.logits) + row * a.ld_logits + c0;
  T* out = a.grad ? static_cast<T*>(a.grad) + row * a.ld_grad + c0 : nullptr;
  if (tid == 0) {
    for (uint32_t p = 0; p < kParts; ++p) mbar_init(&s_full[p], 1u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const int64_t target = target_of(a, row);
  const float scale = a.grad_scale_dev ? a.grad_scale * *a.grad_scale_dev : a.grad_scale;
  const float target_logit = target >= 0 ? Elem<DT>::get(static_cast<const T*>(a.logits)[row * a.ld_logits + target]) : 0.f;

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
  bool landed = true;

  float m = kNegInf;                             // (a NaN is passed over here and turns up in the sum)
  for (uint32_t i = kept + tid; i < n_vec; i += kRowThreads) {
    float f[V];
    Vec<DT>::get(__ldcs(x_vec + i), f);
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) m = fmaxf(m, f[j]);
  }
  for (uint32_t e = tid; e < rest; e += kRowThreads) m = fmaxf(m, Elem<DT>::get(x[e < head ? e : body + (e - head)]));
  const int never = 0;
  for (uint32_t p = 0; p < kParts; ++p) {
    landed = landed && mbar_wait(&s_full[p], 0u, &never);
    const uint32_t v1 = min((p + 1) * part, kept);
    for (uint32_t i = p * part + tid; i < v1; i += kRowThreads) {
      float f[V];
      Vec<DT>::get(held_vec[i], f);
#pragma unroll
      for (uint32_t j = 0; j < V; ++j) m = fmaxf(m, f[j]);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
  if ((tid & 31u) == 0u) s_warp[tid >> 5][0] = m;
  __syncthreads();
#pragma unroll
  for (uint32_t w = 0; w < kRowThreads / 32; ++w) m = fmaxf(m, s_warp[w][0]);

  float s = landed ? 0.f : NAN;                  // (a copy that never came: the row's results say so)
  const float base = m == kNegInf ? 0.f : m;     // (nothing but masked classes here: every term is exp(-inf) = 0, or a NaN)
  for (uint32_t i = tid; i < n_vec; i += kRowThreads) {
    const uint4 q = i < kept ? held_vec[i] : __ldcs(x_vec + i);
    float f[V], part = 0.f;
    Vec<DT>::get(q, f);
#pragma unroll
    for (uint32_t j = 0; j < V; ++j) part += exp_of(f[j] - base);
    s += part;
  }
  for (uint32_t e = tid; e < rest; e += kRowThreads) s += exp_of(Elem<DT>::get(x[e < head ? e : body + (e - head)]) - base);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  if ((tid & 31u) == 0u) s_warp[tid >> 5][1] = s;
  __syncthreads();
  s = 0.f;
#pragma unroll
  for (uint32_t w = 0; w < kRowThreads / 32; ++w) s += s_warp[w][1];
  if (cluster > 1) {
    if (tid == 0) s_pair = make_float2(m, s);
    cluster_arrive();
    cluster_wait();
    m = kNegInf, s = 0.f;
    for (uint32_t r = 0; r < cluster; ++r) {
      const float2 p = peer_load2(peer_address(smem_u32(&s_pair), r));
      join(m, s, p.x, p.y);
    }
    cluster_arrive();                            // the pairs have been read; waited for before this CTA ends
  }
  const RowResult r = finish(m, s, target, target_logit, scale);
  if (tid == 0 && rank == 0) {
    if (a.loss) a.loss[row] = r.loss;
    if (a.lse) a.lse[row] = r.lse;
  }
  if (out) {
    const uint32_t hit = target >= (int64_t)c0 && target < (int64_t)c1 ? (uint32_t)(target - c0) : 0xFFFFFFFFu;
    const bool none = target == -1;              // 0 whatever the logits: not 0 * NaN
    for (uint32_t i = tid; i < n_vec; i += kRowThreads) {
      const uint4 q = i < kept ? held_vec[i] : __ldcs(x_vec + i);
      float f[V];
      Vec<DT>::get(q, f);
      const uint32_t e0 = head + i * V;
#pragma unroll
      for (uint32_t j = 0; j < V; ++j) f[j] = none ? 0.f : exp_of(f[j] - m) * r.factor;
      if (hit - e0 < V) {
#pragma unroll
        for (uint32_t j = 0; j < V; ++j) f[j] -= e0 + j == hit ? r.scale : 0.f;
      }
      __stcs(reinterpret_cast<uint4*>(out + head) + i, Vec<DT>::put(f));
    }
    for (uint32_t i = tid; i < rest; i += kRowThreads) {
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
  const uint32_t stage = min(slice * item, kMaxStage) / item;
  const size_t smem = (size_t)stage * item;
  static PerDeviceInt ready;
  int dev;
  if (!ready.get(&dev)) {
    const cudaError_t e = cudaFuncSetAttribute(xent_row_kernel<DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxStage);
    if (e != cudaSuccess) return e;
    ready.set(dev, 1);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((uint32_t)(a.rows * cluster));
  cfg.blockDim = dim3(kRowThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, xent_row_kernel<DT>, a, cluster, slice, stage);
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
