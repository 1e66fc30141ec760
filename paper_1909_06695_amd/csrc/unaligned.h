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

// Which columns of a row of D a lane owns: strips of up to LANES lanes, P columns a lane.  The last lane of a row that is no
// whole number of P moves back to the last P columns and shares some with the lane before it, which computes the same values; the two
// are always lanes of one strip (a last strip of a single lane takes its neighbour over), so that what is read, changed and written
// belongs to one workgroup.  Rows of fewer than P columns have one lane and go element by element (WHOLE false).
constexpr int STRIP_LANES = 8;                              // of 16 bytes a lane: 128 bytes
struct LaneColumns {
  int col;
  int n;                                                   // 0, or the columns owned: P (WHOLE) or D
};
template <int P, int LANES = STRIP_LANES> __host__ __device__ __forceinline__ int strip_count(int D) {
  return ((D + P - 1) / P + LANES - 1) / LANES;
}
template <int P, bool WHOLE, int LANES = STRIP_LANES> __device__ __forceinline__ LaneColumns lane_columns(int strip, int lane, int D) {
  if (!WHOLE) return {0, lane == 0 ? D : 0};
  const int lanes = (D + P - 1) / P, strips = strip_count<P, LANES>(D);
  int l = strip * LANES + lane;
  if (lanes > 1 && lanes % LANES == 1) {
    if (strip == strips - 1) l = lane < 2 ? lanes - 2 + lane : lanes;
    else if (l == lanes - 2) l = lanes;
  }
  return {min(l * P, D - P), l < lanes ? P : 0};
}
// N neighbouring columns of a row as fp32, of which the first `n` exist; the others are left alone (load) and not written
// (store).  WHOLE: n is 0 or N, else 0 to N - 1.
template <typename T, int N, bool WHOLE> __device__ __forceinline__ void load_columns(const T* p, float* out, int n) {
  if (WHOLE) {
    if (n == 0) return;
    T v[N];
    load_unaligned<T, N>(p, v);
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = to_f32(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) out[i] = to_f32(p[i]);
  }
}
// The same as it lies in memory, for loads that wait in registers.
template <typename T, int N, bool WHOLE> __device__ __forceinline__ void load_raw_columns(const T* p, UnalignedPack<T, N>& out, int n) {
  if (WHOLE) {
    if (n) out = *reinterpret_cast<const UnalignedPack<T, N>*>(p);
  } else {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) out.v[i] = p[i];
  }
}
template <typename T, int N, bool WHOLE> __device__ __forceinline__ void store_columns(T* p, const float* in, int n) {
  if (WHOLE) {
    if (n == 0) return;
    T v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = from_f32<T>(in[i]);
    store_unaligned<T, N>(p, v);
  } else {
#pragma unroll
    for (int i = 0; i < N - 1; ++i)
      if (i < n) p[i] = from_f32<T>(in[i]);
  }
}

}  // namespace ouro
