// Gated linear recurrence h_t = f_t h_{t-1} + (1 - f_t) x_t, f_t = sigmoid(z_t), forward and backward.
//
// A step is the affine map h -> f h + u with u = (1 - f) x, and maps compose: (A, H) after (a, h) is (A a, A h + H).  So a thread
// takes eight consecutive steps (backward four) of four channels and composes their maps, the rows of a wave and then the waves of a workgroup
// scan over these, and with the state that enters its steps known each thread runs them once more from registers.
// Backward, with G_t = dh_t + f_{t+1} G_{t+1} and P_t = f_t G_t: P_t = f_t P_{t+1} + f_t dh_t, the same kind of map from the right with the
// same factors; dx_t = (1 - f_t) G_t, dz_t = G_t (h_{t-1} - x_t) f_t (1 - f_t).  h is formed again from the fp32 states that the forward
// pass left at every 64th step, so that it is neither read back nor rounded.
//
// Bound by memory: z, x (and dh) read once, h (or dz, dx) written once.  A workgroup owns 128 bytes of channels of one stream and a
// tile of steps (256 in bf16, 512 in fp32, backward half of that).  Where streams and channels fill the chip it walks over its tiles itself.  Where they do not,
// every tile has a workgroup: it publishes its map, reads those of up to RC_BACK tiles before it and the state behind the tile
// before these, and publishes the state behind itself.  Tiles are dealt by a counter, so that a workgroup only waits for
// workgroups that have begun before it and every wait ends.  Nothing is read twice.
#include "common.h"
#include "unaligned.h"

#include <algorithm>

namespace ouro {

constexpr int RC_WAVES = 8;                                // most waves of a workgroup
constexpr int RC_BACK = 8;                                 // tiles whose maps a workgroup looks back over
constexpr int RC_TICKET_BYTES = 64;
constexpr int RC_P = 4;                                    // channels of a lane
constexpr int RC_FWD = 8, RC_BWD = 4;                      // and consecutive steps: as many as let two workgroups share a CU (128 registers)
template <typename T, int STEPS_OF_LANE = RC_FWD> struct RcShape {
  static constexpr int L = STEPS_OF_LANE;
  static constexpr int LANES = 128 / (RC_P * (int)sizeof(T)), ROWS = 64 / LANES;       // of a wave
  static constexpr int W = LANES * RC_P;                   // channels of a workgroup
  static constexpr int STEPS = ROWS * L;                // steps of a wave
};
constexpr int RC_KEEP = RECURRENCE_STRIDE;
static_assert(RC_KEEP % RcShape<float, RC_BWD>::STEPS == 0 && RC_KEEP % RcShape<bf16_t, RC_BWD>::STEPS == 0 && RC_KEEP % RC_FWD == 0, "a kept state every whole number of waves");

struct RecurrenceParams {
  int B, T, D, strips, tiles;
  const void* z; const void* x; const void* dh;
  size_t ldz, ldx, lddh;
  const float* h0; const float* dhT; const int32_t* lens;
  void* h; void* dz; void* dx;
  size_t ldh, lddz, lddx;
  float* hT; float* dh0; float* states;
  unsigned* ticket;
  unsigned long long* maps;                                // [tile][B][D]: the map of a tile, factor below, offset above; 0: not there yet
  unsigned* behind;                                        // [tile][B][D]: the state behind a tile; 0: not there yet
};

// Published numbers are stored inverted, with one pattern for all NaN: then 0, which the workspace is cleared to, is none of them.  A
// number is its own flag, so that no order between two stores matters.
__device__ __forceinline__ unsigned rc_code(float v) { return v != v ? ~0x7fc00000u : ~__float_as_uint(v); }
__device__ __forceinline__ float rc_value(unsigned c) { return __uint_as_float(~c); }
template <typename U> __device__ __forceinline__ U rc_peek(const U* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename U> __device__ __forceinline__ void rc_post(U* p, U v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// f and 1 - f from one exponential, neither by subtraction; z = +-infinity gives exactly 1 and 0, NaN gives NaN.
__device__ __forceinline__ void rc_gate(float z, float& f, float& e) {
  const float t = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(z)), r = __builtin_amdgcn_rcpf(1.f + t), q = t * r;
  f = z >= 0.f ? r : q;
  e = z >= 0.f ? q : r;
}

// What a thread needs to find its elements.
struct RcPlace {
  int b, col, ncol, wave, row, lane, waves, len;
  size_t base;                                             // row of step 0
  size_t state;                                            // element of the first channel in [B][D]
};
template <typename T, bool WHOLE>
__device__ __forceinline__ RcPlace rc_place(const RecurrenceParams& p, int strip, int b) {
  RcPlace a;
  a.b = b;
  a.lane = threadIdx.x % RcShape<T>::LANES;
  a.row = (threadIdx.x & 63) / RcShape<T>::LANES;
  a.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  a.waves = blockDim.x >> 6;
  const LaneColumns own = lane_columns<RC_P, WHOLE, RcShape<T>::LANES>(strip, a.lane, p.D);
  a.col = own.n ? own.col : 0;
  a.ncol = own.n;
  a.len = p.lens ? max(0, min(p.T, p.lens[b])) : p.T;
  a.base = (size_t)b * p.T;
  a.state = (size_t)b * p.D + a.col;
  return a;
}

// The four columns of a lane as they lie in memory.
template <typename T> struct RcRaw {
  typedef uint32_t Words __attribute__((ext_vector_type(RC_P * sizeof(T) / 4)));
  union { Words w; T v[RC_P]; };
};
// Row t of an operand at the lane's columns.
template <typename T> __device__ __forceinline__ size_t rc_at(const RcPlace& a, size_t ld, int t) { return (a.base + (unsigned)t) * ld + a.col; }
// The rows [t, t + L); `none` for steps that are not taken.  Loads are not predicated: a step past the end reads the last row (and a lane
// without columns the first ones), and what it finds is replaced.
template <typename T, bool WHOLE, int L>
__device__ __forceinline__ void rc_load(const RecurrenceParams& p, const RcPlace& a, const void* from, size_t ld, int t, float none, RcRaw<T> (&v)[L]) {
  typedef typename RcRaw<T>::Words Unaligned __attribute__((aligned(sizeof(T))));
  RcRaw<T> fill;
#pragma unroll
  for (int j = 0; j < RC_P; ++j) fill.v[j] = from_f32<T>(none);
#pragma unroll
  for (int i = 0; i < L; ++i) {
    const T* row = reinterpret_cast<const T*>(from) + rc_at<T>(a, ld, min(t + i, p.T - 1));
    if (WHOLE) {
      v[i].w = *reinterpret_cast<const Unaligned*>(row);
    } else {
      v[i] = fill;
#pragma unroll
      for (int j = 0; j < RC_P - 1; ++j)
        if (j < a.ncol) v[i].v[j] = row[j];
    }
  }
#pragma unroll
  for (int i = 0; i < L; ++i) v[i].w = t + i < a.len ? v[i].w : fill.w;
}
template <typename T, bool WHOLE>
__device__ __forceinline__ void rc_store(const RcPlace& a, void* to, size_t ld, int t, const float (&in)[RC_P]) {
  store_columns<T, RC_P, WHOLE>(reinterpret_cast<T*>(to) + rc_at<T>(a, ld, t), in, a.ncol);
}

// The exclusive scan of (A, H) over the rows of a wave; the last row's inclusive value goes to LDS (sA may be null).  UP: rows below come first.
template <int ROWS, int LANES, bool UP>
__device__ __forceinline__ void rc_wave_scan(const RcPlace& a, float (&A)[RC_P], float (&H)[RC_P], float* sA, float* sH) {
#pragma unroll
  for (int o = 1; o < ROWS; o <<= 1) {
    const bool on = UP ? a.row >= o : a.row + o < ROWS;
#pragma unroll
    for (int j = 0; j < RC_P; ++j) {
      const float pa = UP ? __shfl_up(A[j], o * LANES, 64) : __shfl_down(A[j], o * LANES, 64);
      const float ph = UP ? __shfl_up(H[j], o * LANES, 64) : __shfl_down(H[j], o * LANES, 64);
      if (on) { H[j] = fmaf(A[j], ph, H[j]); A[j] *= pa; }
    }
  }
  if (a.row == (UP ? ROWS - 1 : 0)) {
#pragma unroll
    for (int j = 0; j < RC_P; ++j) { if (sA) sA[j] = A[j]; sH[j] = H[j]; }
  }
#pragma unroll
  for (int j = 0; j < RC_P; ++j) {
    const float pa = UP ? __shfl_up(A[j], LANES, 64) : __shfl_down(A[j], LANES, 64);
    const float ph = UP ? __shfl_up(H[j], LANES, 64) : __shfl_down(H[j], LANES, 64);
    const bool on = UP ? a.row > 0 : a.row + 1 < ROWS;
    A[j] = on ? pa : 1.f;
    H[j] = on ? ph : 0.f;
  }
}

// The state that enters tile `nth` in the order of the scan, in every thread, given the tile's own map (A, H).  `from`: h0 or dhT.
// The first tile publishes a map that holds the state before it (factor 0), which later tiles therefore do not read.  The rows of
// the first wave look back over RC_BACK / ROWS tiles each and compose what they find like steps.
template <typename T, bool WHOLE>
__device__ __forceinline__ void rc_enter(const RecurrenceParams& p, const RcPlace& a, int nth, const float* from, const float (&A)[RC_P], const float (&H)[RC_P],
                                         float (&state)[RC_P], float* shared) {
  constexpr int ROWS = RcShape<T>::ROWS, LANES = RcShape<T>::LANES, PER = RC_BACK / ROWS;
  const size_t stride = (size_t)p.B * p.D;                 // of tiles
  if (a.wave == 0) {
    float f[RC_P], h[RC_P];                                // the map from what precedes the row's tiles to what follows them
#pragma unroll
    for (int j = 0; j < RC_P; ++j) { f[j] = 1.f; h[j] = 0.f; }
    if (nth == 0 && from) load_columns<float, RC_P, WHOLE>(from + a.state, h, a.ncol);
    if (a.row == 0 && nth + 1 < p.tiles)
#pragma unroll
      for (int j = 0; j < RC_P; ++j)
        if (j < a.ncol)
          rc_post(p.maps + nth * stride + a.state + j,
                  (unsigned long long)rc_code(nth == 0 ? fmaf(A[j], h[j], H[j]) : H[j]) << 32 | rc_code(nth == 0 ? 0.f : A[j]));
    if (nth > 0) {
      const int m0 = max(0, nth - RC_BACK);                // the first tile looked at; the state behind the one before it is there, too
      const int mine = m0 + a.row * PER;
      unsigned long long m[PER][RC_P];
      unsigned c[RC_P];
      bool wait = true;
      while (wait) {                                       // what is there stays there
        wait = false;
#pragma unroll
        for (int j = 0; j < RC_P; ++j) {
          c[j] = 1;
          if (j < a.ncol && a.row == 0 && m0 > 0) c[j] = rc_peek(p.behind + (m0 - 1) * stride + a.state + j);
          wait |= c[j] == 0;
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            m[i][j] = 1;
            if (j < a.ncol && mine + i < nth) m[i][j] = rc_peek(p.maps + (mine + i) * stride + a.state + j);
            wait |= m[i][j] == 0;
          }
        }
        wait = __any(wait);
        if (wait) __builtin_amdgcn_s_sleep(1);
      }
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        if (a.row == 0 && m0 > 0) { f[j] = 0.f; h[j] = rc_value(c[j]); }
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (mine + i < nth) {
            const float mf = rc_value((unsigned)m[i][j]), mh = rc_value((unsigned)(m[i][j] >> 32));
            h[j] = mine + i == 0 ? mh : fmaf(mf, h[j], mh);
            f[j] *= mf;
          }
      }
#pragma unroll
      for (int o = 1; o < ROWS; o <<= 1)
#pragma unroll
        for (int j = 0; j < RC_P; ++j) {
          const float pf = __shfl_up(f[j], o * LANES, 64), ph = __shfl_up(h[j], o * LANES, 64);
          if (a.row >= o) { h[j] = fmaf(f[j], ph, h[j]); f[j] *= pf; }
        }
    }
    if (a.row == (nth > 0 ? ROWS - 1 : 0)) {
      if (nth + 1 < p.tiles && p.tiles > RC_BACK + 1)
#pragma unroll
        for (int j = 0; j < RC_P; ++j)
          if (j < a.ncol) rc_post(p.behind + nth * stride + a.state + j, rc_code(fmaf(A[j], h[j], H[j])));
#pragma unroll
      for (int j = 0; j < RC_P; ++j) shared[a.lane * RC_P + j] = h[j];
    }
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < RC_P; ++j) state[j] = shared[a.lane * RC_P + j];
}

// The strip, stream and (chained) tile of a workgroup.
struct RcWork { int strip, b, nth; };
template <bool CHAINED>
__device__ __forceinline__ RcWork rc_work(const RecurrenceParams& p, unsigned* shared) {
  unsigned w = blockIdx.x;
  if (CHAINED) {
    if (threadIdx.x == 0) *shared = atomicAdd(p.ticket, 1u);
    __syncthreads();
    w = (unsigned)__builtin_amdgcn_readfirstlane((int)*shared);
  }
  const unsigned lines = (unsigned)p.strips * p.B, line = w % lines;
  return {(int)(line % p.strips), (int)(line / p.strips), (int)(w / lines)};
}

// WHOLE: see lane_columns.  CHAINED: a workgroup a tile.
template <typename T, bool WHOLE, bool CHAINED>
__global__ __launch_bounds__(64 * RC_WAVES, 4) void recurrence_fwd_kernel(RecurrenceParams p) {
  using S = RcShape<T>;
  __shared__ float sA[2][RC_WAVES][S::W], sH[2][RC_WAVES][S::W], enter[S::W];
  __shared__ unsigned ticket;
  const RcWork work = rc_work<CHAINED>(p, &ticket);
  const RcPlace a = rc_place<T, WHOLE>(p, work.strip, work.b);
  const int steps = a.waves * S::STEPS;
  float state[RC_P] = {};                                  // what enters the tile
  if (!CHAINED && p.h0) load_columns<float, RC_P, WHOLE>(p.h0 + a.state, state, a.ncol);
  int buf = 0, nth = work.nth;
  do {
    const int tw = nth * steps + a.wave * S::STEPS, t = tw + a.row * S::L;
    float f[S::L][RC_P], u[S::L][RC_P], A[RC_P], H[RC_P];
    {
      RcRaw<T> z[S::L], x[S::L];
      rc_load<T, WHOLE>(p, a, p.z, p.ldz, t, INFINITY, z);    // a step that is not taken keeps the state
      rc_load<T, WHOLE>(p, a, p.x, p.ldx, t, 0.f, x);
#pragma unroll
      for (int j = 0; j < RC_P; ++j) { A[j] = 1.f; H[j] = 0.f; }
#pragma unroll
      for (int i = 0; i < S::L; ++i)
#pragma unroll
        for (int j = 0; j < RC_P; ++j) {
          float e;
          rc_gate(to_f32(z[i].v[j]), f[i][j], e);
          u[i][j] = e * to_f32(x[i].v[j]);
          A[j] *= f[i][j];
          H[j] = fmaf(f[i][j], H[j], u[i][j]);
        }
    }
    rc_wave_scan<S::ROWS, S::LANES, true>(a, A, H, &sA[buf][a.wave][a.lane * RC_P], &sH[buf][a.wave][a.lane * RC_P]);
    __syncthreads();
    float before_a[RC_P], before_h[RC_P], all_a[RC_P], all_h[RC_P];            // the maps of the waves before this one, and of the tile
#pragma unroll
    for (int j = 0; j < RC_P; ++j) { all_a[j] = 1.f; all_h[j] = 0.f; }
    for (int w = 0; w < a.waves; ++w)
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        if (w == a.wave) { before_a[j] = all_a[j]; before_h[j] = all_h[j]; }
        const float m = sA[buf][w][a.lane * RC_P + j];
        all_h[j] = fmaf(m, all_h[j], sH[buf][w][a.lane * RC_P + j]);
        all_a[j] *= m;
      }
    if (CHAINED) rc_enter<T, WHOLE>(p, a, nth, p.h0, all_a, all_h, state, enter);
    float h[RC_P];
#pragma unroll
    for (int j = 0; j < RC_P; ++j) {
      h[j] = fmaf(A[j], fmaf(before_a[j], state[j], before_h[j]), H[j]);
      state[j] = fmaf(all_a[j], state[j], all_h[j]);
    }
    if (p.states && t % RC_KEEP == 0 && t < p.T)
      store_columns<float, RC_P, WHOLE>(p.states + ((size_t)a.b * ((p.T + RC_KEEP - 1) / RC_KEEP) + t / RC_KEEP) * p.D + a.col, h, a.ncol);
#pragma unroll
    for (int i = 0; i < S::L; ++i) {
#pragma unroll
      for (int j = 0; j < RC_P; ++j) h[j] = fmaf(f[i][j], h[j], u[i][j]);
      float out[RC_P];
#pragma unroll
      for (int j = 0; j < RC_P; ++j) out[j] = t + i < a.len ? h[j] : 0.f;
      if (t + i < p.T) rc_store<T, WHOLE>(a, p.h, p.ldh, t + i, out);
    }
    buf ^= 1;
  } while (++nth < p.tiles && !CHAINED);
  if (nth == p.tiles && a.wave == 0 && a.row == 0 && p.hT) store_columns<float, RC_P, WHOLE>(p.hT + a.state, state, a.ncol);
}

// Tiles from the last one on.
template <typename T, bool WHOLE, bool CHAINED>
__global__ __launch_bounds__(64 * RC_WAVES, 4) void recurrence_bwd_kernel(RecurrenceParams p) {
  using S = RcShape<T, RC_BWD>;
  __shared__ float sA[2][RC_WAVES][S::W], sH[2][RC_WAVES][S::W], sQ[2][RC_WAVES][S::W], enter[S::W];
  __shared__ unsigned ticket;
  const RcWork work = rc_work<CHAINED>(p, &ticket);
  const RcPlace a = rc_place<T, WHOLE>(p, work.strip, work.b);
  const int steps = a.waves * S::STEPS;
  float state[RC_P] = {};                                  // P of the step behind the tile
  if (!CHAINED && p.dhT) load_columns<float, RC_P, WHOLE>(p.dhT + a.state, state, a.ncol);
  int buf = 0, nth = work.nth;
  do {
    const int tw = (p.tiles - 1 - nth) * steps + a.wave * S::STEPS, t = tw + a.row * S::L;
    RcRaw<T> g[S::L];
    // The smaller of f and 1 - f with the sign of z (both follow from it: 1 - it is exact to half a step of a number above a half);
    // x, then h_{t-1} - x_t.
    float s[S::L][RC_P], v[S::L][RC_P], kept[RC_P] = {};
    float A[RC_P], H[RC_P], B[RC_P], Q[RC_P];
    auto gates = [&](float& q, float& f, float& e) __attribute__((always_inline)) {
      asm("" : "+v"(q));                                   // the compiler would keep both numbers of every step from the first time on
      const float small = fabsf(q), large = 1.f - small;
      const bool keep = __float_as_uint(q) >> 31 == 0;
      f = keep ? large : small;
      e = keep ? small : large;
    };
    {
      RcRaw<T> z[S::L], x[S::L];
      rc_load<T, WHOLE>(p, a, p.z, p.ldz, t, INFINITY, z);
      rc_load<T, WHOLE>(p, a, p.x, p.ldx, t, 0.f, x);
      rc_load<T, WHOLE>(p, a, p.dh, p.lddh, t, 0.f, g);
      if (tw < p.T) load_columns<float, RC_P, WHOLE>(p.states + ((size_t)a.b * ((p.T + RC_KEEP - 1) / RC_KEEP) + tw / RC_KEEP) * p.D + a.col, kept, a.ncol);
#pragma unroll
      for (int j = 0; j < RC_P; ++j) { A[j] = 1.f; H[j] = Q[j] = 0.f; }
#pragma unroll
      for (int i = 0; i < S::L; ++i)
#pragma unroll
        for (int j = 0; j < RC_P; ++j) {
          const float zz = to_f32(z[i].v[j]), r = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(zz));
          s[i][j] = copysignf(r * __builtin_amdgcn_rcpf(1.f + r), zz);
          v[i][j] = to_f32(x[i].v[j]);
          float f, e;
          gates(s[i][j], f, e);
          A[j] *= f;
          H[j] = fmaf(f, H[j], e * v[i][j]);
        }
    }
#pragma unroll
    for (int i = S::L - 1; i >= 0; --i)
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        float f, e;
        gates(s[i][j], f, e);
        Q[j] = f * (to_f32(g[i].v[j]) + Q[j]);
      }
#pragma unroll
    for (int j = 0; j < RC_P; ++j) B[j] = A[j];
    rc_wave_scan<S::ROWS, S::LANES, false>(a, B, Q, &sA[buf][a.wave][a.lane * RC_P], &sQ[buf][a.wave][a.lane * RC_P]);
    rc_wave_scan<S::ROWS, S::LANES, true>(a, A, H, nullptr, &sH[buf][a.wave][a.lane * RC_P]);
    __syncthreads();
    float before_a[RC_P], before_q[RC_P], all_a[RC_P], all_q[RC_P];            // the maps of the waves behind this one, and of the tile
#pragma unroll
    for (int j = 0; j < RC_P; ++j) { all_a[j] = 1.f; all_q[j] = 0.f; }
    for (int w = a.waves - 1; w >= 0; --w)
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        if (w == a.wave) { before_a[j] = all_a[j]; before_q[j] = all_q[j]; }
        const float m = sA[buf][w][a.lane * RC_P + j];
        all_q[j] = fmaf(m, all_q[j], sQ[buf][w][a.lane * RC_P + j]);
        all_a[j] *= m;
      }
    // the state that enters the wave: kept, or one or more waves behind a kept one
    for (int w = a.wave - (tw % RC_KEEP) / S::STEPS; w < a.wave; ++w)
#pragma unroll
      for (int j = 0; j < RC_P; ++j) kept[j] = fmaf(sA[buf][w][a.lane * RC_P + j], kept[j], sH[buf][w][a.lane * RC_P + j]);
    if (CHAINED) rc_enter<T, WHOLE>(p, a, nth, p.dhT, all_a, all_q, state, enter);
    float h[RC_P], q[RC_P];
#pragma unroll
    for (int j = 0; j < RC_P; ++j) {
      h[j] = fmaf(A[j], kept[j], H[j]);
      q[j] = fmaf(B[j], fmaf(before_a[j], state[j], before_q[j]), Q[j]);
      state[j] = fmaf(all_a[j], state[j], all_q[j]);
    }
#pragma unroll
    for (int i = 0; i < S::L; ++i)
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        float f, e;
        gates(s[i][j], f, e);
        const float x = v[i][j];
        v[i][j] = h[j] - x;
        h[j] = fmaf(f, h[j], e * x);
      }
#pragma unroll
    for (int i = S::L - 1; i >= 0; --i) {
      float dx[RC_P], dz[RC_P];
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        float f, e;
        gates(s[i][j], f, e);
        const float G = to_f32(g[i].v[j]) + q[j];
        dx[j] = e * G;
        dz[j] = G * v[i][j] * (f * e);
        q[j] = f * G;
        if (t + i >= a.len) dx[j] = dz[j] = 0.f;
      }
      if (t + i < p.T) {
        rc_store<T, WHOLE>(a, p.dx, p.lddx, t + i, dx);
        rc_store<T, WHOLE>(a, p.dz, p.lddz, t + i, dz);
      }
    }
    buf ^= 1;
  } while (++nth < p.tiles && !CHAINED);
  if (nth == p.tiles && a.wave == 0 && a.row == 0 && p.dh0) store_columns<float, RC_P, WHOLE>(p.dh0 + a.state, state, a.ncol);
}

// How a call is laid out: a workgroup a tile where strips and streams alone are fewer workgroups than the chip holds (two a CU).
struct RcPlan { int strips, waves, tiles, chained; };
static RcPlan rc_plan(int dtype, bool backward, int B, int T, int D) {
  RcPlan r;
  const int steps = (dtype == 1 ? RcShape<bf16_t>::ROWS : RcShape<float>::ROWS) * (backward ? RC_BWD : RC_FWD);
  r.strips = dtype == 1 ? strip_count<RC_P, RcShape<bf16_t>::LANES>(D) : strip_count<RC_P, RcShape<float>::LANES>(D);
  r.waves = 1;
  while (r.waves < RC_WAVES && (long long)r.waves * steps < T) r.waves *= 2;
  r.tiles = (int)(((long long)T + r.waves * steps - 1) / (r.waves * steps));
  r.chained = r.tiles > 1 && (long long)B * r.strips < 512;
  return r;
}
static size_t rc_map_count(const RcPlan& r, int B, int D) { return (size_t)r.tiles * B * D; }
static size_t rc_scratch_bytes(const RcPlan& r, int B, int D) { return r.chained ? RC_TICKET_BYTES + (rc_map_count(r, B, D) * 12 + 15) / 16 * 16 : 0; }
size_t recurrence_scratch_floats(int B, int T, int D) {
  size_t n = 0;
  for (int i = 0; i < 4; ++i) n = std::max(n, rc_scratch_bytes(rc_plan(i & 1, i > 1, B, T, D), B, D));
  return n / 4;
}

template <typename T, bool WHOLE, bool CHAINED>
static void rc_launch(hipStream_t s, unsigned blocks, int waves, const RecurrenceParams& p, bool backward) {
  if (backward) hipLaunchKernelGGL((recurrence_bwd_kernel<T, WHOLE, CHAINED>), dim3(blocks), dim3(64 * waves), 0, s, p);
  else hipLaunchKernelGGL((recurrence_fwd_kernel<T, WHOLE, CHAINED>), dim3(blocks), dim3(64 * waves), 0, s, p);
}
template <typename T>
static void rc_launch(hipStream_t s, unsigned blocks, const RcPlan& plan, const RecurrenceParams& p, bool backward) {
  if (p.D >= RC_P) {
    if (plan.chained) rc_launch<T, true, true>(s, blocks, plan.waves, p, backward);
    else rc_launch<T, true, false>(s, blocks, plan.waves, p, backward);
  } else {
    if (plan.chained) rc_launch<T, false, true>(s, blocks, plan.waves, p, backward);
    else rc_launch<T, false, false>(s, blocks, plan.waves, p, backward);
  }
}
hipError_t launch_recurrence(hipStream_t s, int dtype, const RecurrenceDesc& r) {
  const bool backward = r.dz != nullptr;
  const RcPlan plan = rc_plan(dtype, backward, r.B, r.T, r.D);
  const long long blocks = (long long)r.B * plan.strips * (plan.chained ? plan.tiles : 1);
  if (blocks * 64 * plan.waves >> 32 || (plan.chained && !r.scratch)) return hipErrorInvalidValue;
  RecurrenceParams p;
  memset(&p, 0, sizeof p);
  p.B = r.B; p.T = r.T; p.D = r.D; p.strips = plan.strips; p.tiles = plan.tiles;
  p.z = r.z; p.x = r.x; p.dh = r.dh; p.ldz = r.ldz; p.ldx = r.ldx; p.lddh = r.lddh;
  p.h0 = r.h0; p.dhT = r.dhT; p.lens = r.lens;
  p.h = r.h; p.dz = r.dz; p.dx = r.dx; p.ldh = r.ldh; p.lddz = r.lddz; p.lddx = r.lddx;
  p.hT = r.hT; p.dh0 = r.dh0; p.states = r.states;
  if (plan.chained) {
    char* at = reinterpret_cast<char*>(r.scratch);
    p.ticket = reinterpret_cast<unsigned*>(at);
    p.maps = reinterpret_cast<unsigned long long*>(at + RC_TICKET_BYTES);
    p.behind = reinterpret_cast<unsigned*>(p.maps + rc_map_count(plan, r.B, r.D));
    const hipError_t e = launch_fill_zero(s, at, rc_scratch_bytes(plan, r.B, r.D));
    if (e != hipSuccess) return e;
  }
  if (dtype == 1) rc_launch<bf16_t>(s, (unsigned)blocks, plan, p, backward);
  else rc_launch<float>(s, (unsigned)blocks, plan, p, backward);
  return hipGetLastError();
}

}  // namespace ouro
