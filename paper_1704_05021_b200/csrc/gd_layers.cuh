// Shared by the layers of include/gd_layers.h: rows of any type and alignment in pieces of V elements, sums over a group of threads.
#pragma once

#include "gd_layers.h"
#include "gd_train.cuh"

namespace gd {

// V neighbours of a row as they lie in memory (V sizeof(T) = 2, 4, 8 or 16 bytes, aligned to that).
template <int BYTES>
struct RawOf;
template <> struct RawOf<2> { using type = uint16_t; };
template <> struct RawOf<4> { using type = uint32_t; };
template <> struct RawOf<8> { using type = uint2; };
template <> struct RawOf<16> { using type = uint4; };
template <int DT, int V>
struct Piece {
  using T = typename Elem<DT>::type;
  using Raw = typename RawOf<V * (int)sizeof(T)>::type;
  static __device__ __forceinline__ Raw none() { return Raw{}; }
  static __device__ __forceinline__ Raw load(const T* p) { return __ldcs(reinterpret_cast<const Raw*>(p)); }      // read once
  static __device__ __forceinline__ Raw load_kept(const T* p) { return *reinterpret_cast<const Raw*>(p); }  // read again soon
  static __device__ __forceinline__ void store(T* p, const Raw& r) { __stcs(reinterpret_cast<Raw*>(p), r); }
  static __device__ __forceinline__ void widen(const Raw& r, float* x) {
    if constexpr (sizeof(T) == 4) {
      const float* f = reinterpret_cast<const float*>(&r);
#pragma unroll
      for (int j = 0; j < V; ++j) x[j] = f[j];
    } else if constexpr (V == 1) {
      x[0] = Elem<DT>::get(*reinterpret_cast<const T*>(&r));
    } else {
      const uint32_t* w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
      for (int j = 0; j < V / 2; ++j) {
        const float2 f = unpack2<DT>(w[j]);
        x[2 * j] = f.x, x[2 * j + 1] = f.y;
      }
    }
  }
  static __device__ __forceinline__ Raw narrow(const float* x) {
    Raw r;
    if constexpr (sizeof(T) == 4) {
      float* f = reinterpret_cast<float*>(&r);
#pragma unroll
      for (int j = 0; j < V; ++j) f[j] = x[j];
    } else if constexpr (V == 1) {
      *reinterpret_cast<T*>(&r) = Elem<DT>::put(x[0]);
    } else {
      uint32_t* w = reinterpret_cast<uint32_t*>(&r);
#pragma unroll
      for (int j = 0; j < V / 2; ++j) w[j] = pack2<DT>(x[2 * j], x[2 * j + 1]);
    }
    return r;
  }
};

// Whether rows of `width` elements of `item` bytes, `ld` apart from p on, can be taken in pieces of `v` elements.
inline bool in_pieces(const void* p, uint64_t ld, uint64_t rows, uint64_t width, size_t item, uint32_t v) {
  return !p || (aligned_to(p, item * v) && width % v == 0 && (rows <= 1 || ld % v == 0));
}
inline bool good_matrix(const void* p, uint64_t ld, uint64_t rows, uint64_t width, size_t item) {
  return p && aligned_to(p, item) && (rows <= 1 || ld >= width) && !(ld >> 40);
}

// Copies of 4, 8 or 16 bytes into shared memory that a thread asks for and waits for by itself.
template <int BYTES>
__device__ __forceinline__ void copy_ahead(uint32_t to, const void* from) {
  if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
  else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int LEFT>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(LEFT) : "memory"); }   // all groups but the last LEFT

// The lanes' sum, the same in all of them.
__device__ __forceinline__ float warp_sum(float s) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xFFFFFFFFu, s, o);
  return s;
}

}  // namespace gd
