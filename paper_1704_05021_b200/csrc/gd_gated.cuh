// The gated block's product: what the host and the two kernels share.
#pragma once

#include "gd_linear.cuh"

namespace gd {

// out[r, c] = act(G) * U and pre[r, c] = G, pre[r, cols + c] = U, with G and U the two projections plus their bias.
struct GatedEpilogue {
  void* out;
  void* pre;
  const void* bias;
  uint64_t ld_out, ld_pre;
  uint32_t rows, cols;
  int32_t dtype, bias_dtype, activation;
  uint32_t vectors;           // cols is a multiple of 8, and all buffers take 16-byte accesses at columns that are
};
struct GatedProduct {
  Operand x, gate, up;        // [rows, depth]; the two halves of W
  uint32_t depth;
  bool bf16;
  GatedEpilogue ep;
  int* status;
};
cudaError_t launch_gated_product(const GatedProduct& p, cudaStream_t stream);

// act(g) * u in g's place.
template <int N>
__device__ __forceinline__ void gate_all(float* g, const float* u, int act) {
  activate_all<N>(g, act);
#pragma unroll
  for (int j = 0; j < N; ++j) g[j] *= u[j];
}

}  // namespace gd
