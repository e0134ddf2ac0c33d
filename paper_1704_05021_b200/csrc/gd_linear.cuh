// Shared by the linear layer and the gated block: ragged operands, the workspace, the products of a backward call.
#pragma once

#include <algorithm>

#include "gd_mma.cuh"

namespace gd {

constexpr uint32_t kStatusBytes = 256;

// ---------------------------------------------------------------- ragged operands
// A matrix of 16-bit elements whose rows are no multiple of 16 bytes (or start anywhere), laid out with rows of 8 `vecs` elements; the
// columns between are zeros.  A thread makes 16 bytes of the result: bound by the bytes, read and written once.
struct Pack {
  const uint16_t* src;
  uint4* dst;
  uint64_t ld;
  uint32_t rows, cols, vecs;
};
struct Packs {
  Pack p[3];
  uint32_t count;
};
__device__ __forceinline__ void pack_rows(const Packs& all, uint64_t first, uint64_t step) {
  for (uint32_t i = 0; i < all.count; ++i) {
    const Pack& k = all.p[i];
    const uint64_t total = (uint64_t)k.rows * k.vecs;
#pragma unroll 4
    for (uint64_t t = first; t < total; t += step) {
      // (64-bit division only where 32 bits do not hold the position)
      const uint32_t r = total >> 32 ? (uint32_t)(t / k.vecs) : (uint32_t)t / k.vecs, c = ((uint32_t)t - r * k.vecs) * 8u;
      const uint16_t* s = k.src + r * k.ld + c;
      uint32_t w[4];
      if (c + 8 <= k.cols && ((uintptr_t)s & 7u) == 0) {
        const uint2 lo = __ldcs(reinterpret_cast<const uint2*>(s)), hi = __ldcs(reinterpret_cast<const uint2*>(s) + 1);
        w[0] = lo.x, w[1] = lo.y, w[2] = hi.x, w[3] = hi.y;
      } else if (c + 8 <= k.cols && ((uintptr_t)s & 3u) == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = reinterpret_cast<const uint32_t*>(s)[j];
      } else {
#pragma unroll
        for (uint32_t j = 0; j < 4; ++j) {
          const uint32_t a = c + 2 * j < k.cols ? s[2 * j] : 0u, b = c + 2 * j + 1 < k.cols ? s[2 * j + 1] : 0u;
          w[j] = a | b << 16;
        }
      }
      k.dst[t] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}
inline uint32_t pack_ctas(const Packs& all, uint32_t threads) {
  uint64_t most = 0;
  for (uint32_t i = 0; i < all.count; ++i) most = std::max(most, ((uint64_t)all.p[i].rows * all.p[i].vecs + threads - 1) / threads);
  return (uint32_t)std::min<uint64_t>(most, (uint64_t)sm_count() * 1024 / threads);
}
cudaError_t launch_pack(const Packs& all, cudaStream_t stream);

// ---------------------------------------------------------------- host side
inline uint64_t up(uint64_t x, uint64_t a) { return (x + a - 1) / a * a; }
inline bool tiles_as_it_is(const void* p, uint64_t ld) { return aligned_to(p, 16) && ld % 8 == 0; }
// 16-byte accesses at columns that are multiples of 8 stay aligned
inline bool vector_rows(const void* p, uint64_t ld, int dt) { return !p || (aligned_to(p, 16) && ld * dtype_bytes(dt) % 16 == 0); }

// 16-bit rows that take 4-byte accesses at even columns
inline bool paired_rows(const void* p, uint64_t ld, int dt) { return !p || (dt != GD_DTYPE_FP32 && aligned_to(p, 4) && ld % 2 == 0); }

struct Workspace {
  unsigned char* base;
  size_t at, size;
  void* take(uint64_t rows, uint64_t cols) {
    unsigned char* p = base + at;
    at += up(rows * up(cols, 8) * 2, 256);
    return at <= size ? p : nullptr;
  }
};
// The partial sums' place, where a contraction is long enough to want one.
inline int partial_place(uint64_t depth, Workspace& ws, float** p) {
  if (depth < kLongDepth) return GD_OK;
  *p = static_cast<float*>(ws.take(1, kPartialBytes / 2));
  return *p ? GD_OK : GD_ERR_WORKSPACE;
}
// A leading dimension for one row is never used: a ragged one would only cause a copy.
inline uint64_t row_step(uint64_t ld, uint64_t rows, uint64_t cols) { return rows > 1 ? ld : up(cols, 8); }

// `p` as an operand the tiled copies can read, added to what has to be laid out in the workspace if need be.
inline int operand(const void* p, uint64_t ld, uint64_t rows, uint64_t cols, Workspace& ws, Packs* packs, Operand* o) {
  o->p = p;
  o->ld = row_step(ld, rows, cols);
  if (rows == 0 || cols == 0 || tiles_as_it_is(p, o->ld)) return GD_OK;
  void* q = ws.take(rows, cols);
  if (!q) return GD_ERR_WORKSPACE;
  packs->p[packs->count++] = Pack{static_cast<const uint16_t*>(p), static_cast<uint4*>(q), ld, (uint32_t)rows, (uint32_t)cols, (uint32_t)((cols + 7) / 8)};
  o->p = q;
  o->ld = up(cols, 8);
  return GD_OK;
}
inline bool good_rows(const void* p, uint64_t ld, uint64_t rows, uint64_t cols, size_t item) {
  return p && aligned_to(p, item) && (rows <= 1 || ld >= cols) && !(ld >> 40);
}
inline int check_workspace(const void* ws, size_t bytes) { return !ws || !aligned_to(ws, 256) || bytes < kStatusBytes ? GD_ERR_WORKSPACE : GD_OK; }

// The products of a backward call: dx = dz W^T and dw = x^T dz (or its transpose), either of them where its buffer is given.
struct BackProducts {
  Operand dz, w, x;           // (what a product does not take is not read)
  float* partial;
  uint64_t m, n, k;           // dz is [m, n], x [m, k]
  bool in_out, add;           // add: to what dw holds
  int dtype, dw_dtype;
  void* dx;
  uint64_t ld_dx;
  void* dw;
  uint64_t ld_dw;
  int* status;
};
cudaError_t launch_back_products(const BackProducts& q, cudaStream_t stream);

}  // namespace gd
