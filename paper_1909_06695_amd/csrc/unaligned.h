// Accesses of up to 16 bytes at any element address.  The type's alignment is declared as the element's, and the compiler
// takes what the target allows: one 16-byte instruction (gfx950 reads and writes global memory at any address).
#pragma once
#include "common.h"

namespace ouro {

template <typename T, int N> struct __attribute__((packed, aligned(sizeof(T)))) UnalignedPack { T v[N]; };

template <typename T, int N> __device__ __forceinline__ void load_unaligned(const T* p, T* out) {
  const UnalignedPack<T, N> u = *reinterpret_cast<const UnalignedPack<T, N>*>(p);
#pragma unroll
  for (int i = 0; i < N; ++i) out[i] = u.v[i];
}
template <typename T, int N> __device__ __forceinline__ void store_unaligned(T* p, const T* in) {
  UnalignedPack<T, N> u;
#pragma unroll
  for (int i = 0; i < N; ++i) u.v[i] = in[i];
  *reinterpret_cast<UnalignedPack<T, N>*>(p) = u;
}

// N neighbouring columns of a row as fp32, of which the first `n` exist; the others are left alone (load) and not written
// (store).  WHOLE: n is 0 or N.
template <typename T, int N, bool WHOLE> __device__ __forceinline__ void load_columns(const T* p, float* out, int n) {
  if (n == N) {
    T v[N];
    load_unaligned<T, N>(p, v);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = to_f32(v[i]);
  } else if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) out[i] = to_f32(p[i]);
  }
}
template <typename T, int N, bool WHOLE> __device__ __forceinline__ void store_columns(T* p, const float* in, int n) {
  if (n == N) {
    T v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = from_f32<T>(in[i]);
    store_unaligned<T, N>(p, v);
  } else if (!WHOLE) {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) p[i] = from_f32<T>(in[i]);
  }
}

}  // namespace ouro
