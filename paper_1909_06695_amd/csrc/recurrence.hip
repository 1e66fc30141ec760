// Gated linear recurrence h_t = f_t h_{t-1} + (1 - f_t) x_t, f_t = sigmoid(z_t), forward and backward.
//
// A step is the affine map h -> f h + u with u = (1 - f) x, and maps compose: (A, H) after (a, h) is (A a, A h + H).  So a thread
// takes eight consecutive steps (backward four) of four channels and composes their maps, the rows of a wave and then the waves of a workgroup
// scan over these, and with the state that enters its steps known each thread runs them once more from registers.
// Backward, with G_t = dh_t + f_{t+1} G_{t+1} and P_t = f_t G_t: P_t = f_t P_{t+1} + f_t dh_t, the same kind of map from the right with the
// same factors; dx_t = (1 - f_t) G_t, dz_t = G_t (h_{t-1} - x_t) f_t (1 - f_t).  h is formed again from the fp32 states that the forward
// pass left at every 64th step, so that it is neither read back nor rounded.  (Recurrences as scans over maps that compose: Blelloch 1990; tiles that publish
// their map, then the state behind them, and look back over those before: Merrill and Garland 2016.)
//
// Bound by memory: z, x (and dh) read once, h (or dz, dx) written once.  A workgroup owns 128 bytes of channels of one stream and a
// tile of steps (256 in bf16, 512 in fp32, backward half of that).  Where streams and channels fill the chip it walks over its tiles itself.  Where they do not,
// every tile has a workgroup: it publishes its map, reads those of up to RC_BACK tiles before it and the state behind the tile
// before these, and publishes the state behind itself.  The tiles of a line (a strip of a stream) are dealt by a counter, so that a
// workgroup only waits for workgroups that have begun before it and every wait ends.  Nothing is read twice.
// 8 streams of 1024 steps, 1024 channels, bf16: forward 16 us (51 MB, 3.2 TB/s), backward 25 us (84 MB, 3.4 TB/s), 2 and 4 of them for clearing the
// workspace; one of 65536 steps, 512 channels, fp32: forward 91 us (405 MB, 4.5 TB/s); 64 single tokens of 1024 channels: 5 us.  32 streams of 1024 steps,
// 1024 channels, bf16, which a workgroup walks over: 36 us (201 MB, 5.6 TB/s: repeated calls find part of it in the memory-side cache) and 92 us (336 MB, 3.7 TB/s).
#include "common.h"
#include "unaligned.h"

#include <algorithm>

namespace ouro {

constexpr int RC_WAVES = 8;                                // most waves of a workgroup
constexpr int RC_BACK = 8;                                 // tiles whose maps a workgroup looks back over
constexpr int RC_TICKET_BYTES = 64;                        // of a line: the tickets of one counter for all, 13 ns each, would delay the last of 512 workgroups by 6 us
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
  unsigned* tickets;                                       // of every line, RC_TICKET_BYTES apart
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

// Both in one register: the smaller of them with the sign of z; 1 - it is the other one to half a step.
__device__ __forceinline__ float rc_pack(float z) {
  const float t = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(z));
  return copysignf(t * __builtin_amdgcn_rcpf(1.f + t), z);
}
__device__ __forceinline__ void rc_unpack(float& s, float& f, float& e) {
  asm("" : "+v"(s));                                       // the compiler would hold both numbers of every step from the first time on
  const float small = fabsf(s), large = 1.f - small;
  const bool keep = __float_as_uint(s) >> 31 == 0;
  f = keep ? large : small;
  e = keep ? small : large;
}

// What a thread needs to find its elements.
struct RcPlace {
  int b, col, ncol, wave, row, lane, waves, len;
  size_t base;                                             // row of step 0
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

// Between the waves of a workgroup the first wave goes on with a channel a lane: the column of lane k is that of channel k % 4 of
// lane k / 4 of the strip.
struct RcChannel {
  bool on;
  size_t state;                                            // element in [B][D]
};
template <typename T, bool WHOLE>
__device__ __forceinline__ RcChannel rc_channel(const RecurrenceParams& p, int strip, int b) {
  const int k = threadIdx.x & 63;
  const LaneColumns own = lane_columns<RC_P, WHOLE, RcShape<T>::LANES>(strip, min(k / RC_P, RcShape<T>::LANES - 1), p.D);
  return {k < RcShape<T>::W && k % RC_P < own.n, (size_t)b * p.D + own.col + k % RC_P};
}
// The state that enters tile `nth` in the order of the scan, given the tile's own map (A, H).  `from`: h0 or dhT.
// The first tile publishes a map that holds the state before it (factor 0), which later tiles therefore do not read.
__device__ __forceinline__ float rc_enter(const RecurrenceParams& p, const RcChannel& c, int nth, const float* from, float A, float H) {
  const size_t stride = (size_t)p.B * p.D;                 // of tiles
  float state = 0.f;
  if (nth == 0) {
    if (c.on && from) state = from[c.state];
    if (c.on && p.tiles > 1) rc_post(p.maps + c.state, (unsigned long long)rc_code(fmaf(A, state, H)) << 32 | rc_code(0.f));
  } else {
    if (c.on && nth + 1 < p.tiles) rc_post(p.maps + nth * stride + c.state, (unsigned long long)rc_code(H) << 32 | rc_code(A));
    const int m0 = max(0, nth - RC_BACK);                  // the first tile looked at; the state behind the one before it is there, too
    unsigned long long m[RC_BACK];
    unsigned before = 1;
    bool wait = true;
    while (wait) {                                         // what is there stays there
      wait = false;
      if (c.on && m0 > 0) wait = (before = rc_peek(p.behind + (m0 - 1) * stride + c.state)) == 0;
#pragma unroll
      for (int i = 0; i < RC_BACK; ++i) {
        m[i] = 1;
        if (c.on && m0 + i < nth) m[i] = rc_peek(p.maps + (m0 + i) * stride + c.state);
      }
#pragma unroll
      for (int i = 0; i < RC_BACK; ++i) wait |= m[i] == 0;
      wait = __any(wait);
      if (wait) __builtin_amdgcn_s_sleep(1);
    }
    if (m0 > 0) state = rc_value(before);
#pragma unroll
    for (int i = 0; i < RC_BACK; ++i)
      if (m0 + i < nth) {
        const float f = rc_value((unsigned)m[i]), h = rc_value((unsigned)(m[i] >> 32));
        state = m0 + i == 0 ? h : fmaf(f, state, h);
      }
  }
  if (c.on && nth + 1 < p.tiles && p.tiles > RC_BACK + 1) rc_post(p.behind + nth * stride + c.state, rc_code(fmaf(A, state, H)));
  return state;
}

// How a stream's tiles are dealt: there is one; a workgroup walks over them; each has a workgroup.
enum { RC_SINGLE, RC_WALK, RC_CHAINED };
// The strip, stream and first tile of a workgroup.
struct RcWork { int strip, b, nth; };
template <int MODE>
__device__ __forceinline__ RcWork rc_work(const RecurrenceParams& p, unsigned* shared) {
  // Workgroups go to the 8 XCDs in turn; an XCD takes neighbouring lines: where rows do not start on cache lines, neighbouring strips
  // share them, and one L2 then fetches and writes them whole.
  const unsigned lines = (unsigned)p.strips * p.B, r = blockIdx.x % lines, xcd = r & 7;
  const unsigned line = xcd * (lines >> 3) + min(xcd, lines & 7) + (r >> 3);
  int nth = 0;
  if (MODE == RC_CHAINED) {
    if (threadIdx.x == 0) *shared = atomicAdd(p.tickets + line * (RC_TICKET_BYTES / 4), 1u);
    __syncthreads();
    nth = __builtin_amdgcn_readfirstlane((int)*shared);
  }
  return {(int)(line % p.strips), (int)(line / p.strips), nth};
}

// WHOLE: see lane_columns.
template <typename T, bool WHOLE, int MODE>
__global__ __launch_bounds__(64 * RC_WAVES, 4) void recurrence_fwd_kernel(RecurrenceParams p) {
  using S = RcShape<T>;
  __shared__ __align__(16) float sA[RC_WAVES][S::W], sH[RC_WAVES][S::W], enter[RC_WAVES][S::W];
  __shared__ unsigned ticket;
  const RcWork work = rc_work<MODE>(p, &ticket);
  const RcPlace a = rc_place<T, WHOLE>(p, work.strip, work.b);
  const RcChannel c = rc_channel<T, WHOLE>(p, work.strip, work.b);
  const int k = min((int)(threadIdx.x & 63), S::W - 1);     // (lanes without a channel read along)
  const bool channel = (int)(threadIdx.x & 63) < S::W;
  const int waves = MODE == RC_SINGLE ? a.waves : RC_WAVES, steps = waves * S::STEPS;
  float carry = 0.f;                                       // first wave, channel k: the state that enters the tile, then the next wave
  if (MODE != RC_CHAINED && a.wave == 0 && c.on && p.h0) carry = p.h0[c.state];
  int nth = work.nth;
  do {
    const int t = nth * steps + a.wave * S::STEPS + a.row * S::L;
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
    rc_wave_scan<S::ROWS, S::LANES, true>(a, A, H, &sA[a.wave][a.lane * RC_P], &sH[a.wave][a.lane * RC_P]);
    __syncthreads();
    if (a.wave == 0) {
      // (what the waves left is read twice rather than held: every register here is one that all steps of the lane live beside)
      if (MODE == RC_CHAINED) {
        float all_a = 1.f, all_h = 0.f;
#pragma unroll
        for (int w = 0; w < RC_WAVES; ++w) { all_h = fmaf(sA[w][k], all_h, sH[w][k]); all_a *= sA[w][k]; }
        carry = rc_enter(p, c, nth, p.h0, all_a, all_h);
      }
      asm volatile("" ::: "memory");
#pragma unroll 4
      for (int w = 0; w < waves; ++w) {
        if (channel) enter[w][k] = carry;
        carry = fmaf(sA[w][k], carry, sH[w][k]);
      }
    }
    __syncthreads();
    float h[RC_P];
#pragma unroll
    for (int j = 0; j < RC_P; ++j) h[j] = fmaf(A[j], enter[a.wave][a.lane * RC_P + j], H[j]);
    if (p.states && t % RC_KEEP == 0 && t < p.T)
      store_columns<float, RC_P, WHOLE>(p.states + ((size_t)a.b * ((p.T + RC_KEEP - 1) / RC_KEEP) + t / RC_KEEP) * p.D + a.col, h, a.ncol);
#pragma unroll
    for (int i = 0; i < S::L; ++i) {
      float out[RC_P];
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        h[j] = fmaf(f[i][j], h[j], u[i][j]);
        out[j] = t + i < a.len ? h[j] : 0.f;
      }
      if (t + i < p.T) rc_store<T, WHOLE>(a, p.h, p.ldh, t + i, out);
    }
  } while (++nth < p.tiles && MODE == RC_WALK);
  if (nth == p.tiles && a.wave == 0 && c.on && p.hT) p.hT[c.state] = carry;
}

// Tiles from the last one on.
template <typename T, bool WHOLE, int MODE>
__global__ __launch_bounds__(64 * RC_WAVES, 4) void recurrence_bwd_kernel(RecurrenceParams p) {
  using S = RcShape<T, RC_BWD>;
  constexpr int KEPT = RC_KEEP / S::STEPS;                 // waves that share a kept state
  __shared__ __align__(16) float sA[RC_WAVES][S::W], sH[RC_WAVES][S::W], sQ[RC_WAVES][S::W], enter[RC_WAVES][S::W], state[RC_WAVES][S::W];
  __shared__ unsigned ticket;
  const RcWork work = rc_work<MODE>(p, &ticket);
  const RcPlace a = rc_place<T, WHOLE>(p, work.strip, work.b);
  const RcChannel c = rc_channel<T, WHOLE>(p, work.strip, work.b);
  const int k = min((int)(threadIdx.x & 63), S::W - 1);     // (lanes without a channel read along)
  const bool channel = (int)(threadIdx.x & 63) < S::W;
  const int waves = MODE == RC_SINGLE ? a.waves : RC_WAVES, steps = waves * S::STEPS;
  float carry = 0.f;                                       // first wave, channel k: P of the step behind the tile, then behind the wave before
  if (MODE != RC_CHAINED && a.wave == 0 && c.on && p.dhT) carry = p.dhT[c.state];
  int nth = work.nth;
  do {
    const int tile = (p.tiles - 1 - nth) * steps, t = tile + a.wave * S::STEPS + a.row * S::L;
    RcRaw<T> g[S::L];
    float s[S::L][RC_P], v[S::L][RC_P];                    // see rc_pack; x, then h_{t-1} - x_t
    float A[RC_P], H[RC_P], B[RC_P], Q[RC_P], kept[RC_WAVES / KEPT];
    const int keeper = waves > 1 ? 1 : 0;                  // the wave that brings in the kept states
    {
      RcRaw<T> z[S::L], x[S::L];
      rc_load<T, WHOLE>(p, a, p.z, p.ldz, t, INFINITY, z);
      rc_load<T, WHOLE>(p, a, p.dh, p.lddh, t, 0.f, g);
      rc_load<T, WHOLE>(p, a, p.x, p.ldx, t, 0.f, x);
      if (a.wave == keeper) {
#pragma unroll
        for (int i = 0; i < RC_WAVES / KEPT; ++i) {
          kept[i] = 0.f;
          if (c.on && tile + i * RC_KEEP < p.T) kept[i] = p.states[((size_t)a.b * ((p.T + RC_KEEP - 1) / RC_KEEP - 1) + tile / RC_KEEP + i) * p.D + c.state];
        }
      }
#pragma unroll
      for (int j = 0; j < RC_P; ++j) { A[j] = 1.f; H[j] = Q[j] = 0.f; }
#pragma unroll
      for (int i = 0; i < S::L; ++i)
#pragma unroll
        for (int j = 0; j < RC_P; ++j) {
          s[i][j] = rc_pack(to_f32(z[i].v[j]));
          v[i][j] = to_f32(x[i].v[j]);
          float f, e;
          rc_unpack(s[i][j], f, e);
          A[j] *= f;
          H[j] = fmaf(f, H[j], e * v[i][j]);
        }
    }
#pragma unroll
    for (int i = S::L - 1; i >= 0; --i)
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        float f, e;
        rc_unpack(s[i][j], f, e);
        Q[j] = f * (to_f32(g[i].v[j]) + Q[j]);
      }
#pragma unroll
    for (int j = 0; j < RC_P; ++j) B[j] = A[j];
    rc_wave_scan<S::ROWS, S::LANES, false>(a, B, Q, &sA[a.wave][a.lane * RC_P], &sQ[a.wave][a.lane * RC_P]);
    rc_wave_scan<S::ROWS, S::LANES, true>(a, A, H, nullptr, &sH[a.wave][a.lane * RC_P]);
    __syncthreads();
    if (a.wave == keeper) {                                // the state that enters a wave: kept, or behind the wave before it
      float h = 0.f;
#pragma unroll
      for (int w = 0; w < RC_WAVES; ++w) {
        h = w % KEPT == 0 ? kept[w / KEPT] : MODE != RC_SINGLE || w < waves ? fmaf(sA[w - 1][k], h, sH[w - 1][k]) : 0.f;
        if (channel) state[w][k] = h;
      }
    }
    if (a.wave == 0) {
      if (MODE == RC_CHAINED) {
        float all_a = 1.f, all_q = 0.f;
#pragma unroll
        for (int w = RC_WAVES - 1; w >= 0; --w) { all_q = fmaf(sA[w][k], all_q, sQ[w][k]); all_a *= sA[w][k]; }
        carry = rc_enter(p, c, nth, p.dhT, all_a, all_q);
      }
      asm volatile("" ::: "memory");
#pragma unroll 4
      for (int w = waves - 1; w >= 0; --w) {
        if (channel) enter[w][k] = carry;
        carry = fmaf(sA[w][k], carry, sQ[w][k]);
      }
    }
    __syncthreads();
    float h[RC_P], q[RC_P];
#pragma unroll
    for (int j = 0; j < RC_P; ++j) {
      h[j] = fmaf(A[j], state[a.wave][a.lane * RC_P + j], H[j]);
      q[j] = fmaf(B[j], enter[a.wave][a.lane * RC_P + j], Q[j]);
    }
#pragma unroll
    for (int i = 0; i < S::L; ++i)
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        const float x = v[i][j];
        v[i][j] = h[j] - x;
        float f, e;
        rc_unpack(s[i][j], f, e);
        h[j] = fmaf(f, h[j], e * x);
      }
#pragma unroll
    for (int i = S::L - 1; i >= 0; --i) {
      float dx[RC_P], dz[RC_P];
#pragma unroll
      for (int j = 0; j < RC_P; ++j) {
        const float G = to_f32(g[i].v[j]) + q[j];
        float f, e;
        rc_unpack(s[i][j], f, e);
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
  } while (++nth < p.tiles && MODE == RC_WALK);
  if (nth == p.tiles && a.wave == 0 && c.on && p.dh0) p.dh0[c.state] = carry;
}

// How a call is laid out: a workgroup a tile where strips and streams alone are fewer workgroups than the chip holds (two a CU).  There walking
// over the tiles needs no workspace and is as fast or faster forward (chained against walking, bf16, 1024 steps and channels: 128 lines 15.7 against
// 20.1 us, 256 lines 26.6 / 23.9, 512 42.8 / 36.1, 1024 94.4 / 93.7; fp32: 256 lines 20.5 / 21.0, 512 37.0 / 32.3), but where streams are long (8192 steps, fp32, 512
// lines: 306 against 364).  Backward it is behind: bf16, 128 lines 26 against 43 us, 256 40 / 46, 512 85 / 92, 768 122 / 156, 1024
// 157 / 173 (512 lines of 300 steps: 31 / 29); fp32, 512 lines 90 / 98.  There the rule buys little but the workspace.
struct RcPlan { int strips, waves, tiles, mode; };
static RcPlan rc_plan(int dtype, bool backward, int B, int T, int D) {
  RcPlan r;
  const int steps = (dtype == 1 ? RcShape<bf16_t>::ROWS : RcShape<float>::ROWS) * (backward ? RC_BWD : RC_FWD);
  r.strips = dtype == 1 ? strip_count<RC_P, RcShape<bf16_t>::LANES>(D) : strip_count<RC_P, RcShape<float>::LANES>(D);
  r.waves = 1;
  while (r.waves < RC_WAVES && (long long)r.waves * steps < T) r.waves *= 2;
  r.tiles = (int)(((long long)T + r.waves * steps - 1) / (r.waves * steps));
  r.mode = r.tiles == 1 ? RC_SINGLE : (long long)B * r.strips < 512 ? RC_CHAINED : RC_WALK;
  return r;
}
static size_t rc_ticket_bytes(const RcPlan& r, int B) { return (size_t)r.strips * B * RC_TICKET_BYTES; }
static size_t rc_map_count(const RcPlan& r, int B, int D) { return (size_t)r.tiles * B * D; }
static size_t rc_scratch_bytes(const RcPlan& r, int B, int D) {
  return r.mode == RC_CHAINED ? rc_ticket_bytes(r, B) + (rc_map_count(r, B, D) * 12 + 15) / 16 * 16 : 0;
}
size_t recurrence_scratch_floats(int B, int T, int D) {
  size_t n = 0;
  for (int i = 0; i < 4; ++i) n = std::max(n, rc_scratch_bytes(rc_plan(i & 1, i > 1, B, T, D), B, D));
  return n / 4;
}

template <typename T, bool WHOLE, int MODE>
static void rc_launch(hipStream_t s, unsigned blocks, int waves, const RecurrenceParams& p, bool backward) {
  if (backward) hipLaunchKernelGGL((recurrence_bwd_kernel<T, WHOLE, MODE>), dim3(blocks), dim3(64 * waves), 0, s, p);
  else hipLaunchKernelGGL((recurrence_fwd_kernel<T, WHOLE, MODE>), dim3(blocks), dim3(64 * waves), 0, s, p);
}
template <typename T, bool WHOLE>
static void rc_launch(hipStream_t s, unsigned blocks, const RcPlan& plan, const RecurrenceParams& p, bool backward) {
  if (plan.mode == RC_SINGLE) rc_launch<T, WHOLE, RC_SINGLE>(s, blocks, plan.waves, p, backward);
  else if (plan.mode == RC_WALK) rc_launch<T, WHOLE, RC_WALK>(s, blocks, plan.waves, p, backward);
  else rc_launch<T, WHOLE, RC_CHAINED>(s, blocks, plan.waves, p, backward);
}
hipError_t launch_recurrence(hipStream_t s, int dtype, const RecurrenceDesc& r) {
  const bool backward = r.dz != nullptr;
  const RcPlan plan = rc_plan(dtype, backward, r.B, r.T, r.D);
  const bool chained = plan.mode == RC_CHAINED;
  if (chained && !r.scratch) return hipErrorInvalidValue;
  RecurrenceParams p;
  memset(&p, 0, sizeof p);
  p.B = r.B; p.T = r.T; p.D = r.D; p.strips = plan.strips; p.tiles = plan.tiles;
  p.z = r.z; p.x = r.x; p.dh = r.dh; p.ldz = r.ldz; p.ldx = r.ldx; p.lddh = r.lddh;
  p.h0 = r.h0; p.dhT = r.dhT; p.lens = r.lens;
  p.h = r.h; p.dz = r.dz; p.dx = r.dx; p.ldh = r.ldh; p.lddz = r.lddz; p.lddx = r.lddx;
  p.hT = r.hT; p.dh0 = r.dh0; p.states = r.states;
  if (chained) {
    char* at = reinterpret_cast<char*>(r.scratch);
    p.tickets = reinterpret_cast<unsigned*>(at);
    p.maps = reinterpret_cast<unsigned long long*>(at + rc_ticket_bytes(plan, r.B));
    p.behind = reinterpret_cast<unsigned*>(p.maps + rc_map_count(plan, r.B, r.D));
    const hipError_t e = launch_fill_zero(s, at, rc_scratch_bytes(plan, r.B, r.D));
    if (e != hipSuccess) return e;
  }
  // A grid has less than 2^32 work items: the tiles of chained lines go into as many launches as that takes, in which the tickets go on
  // (one stream of 2^30 steps in bf16, backward: 2^23 tiles of 512 threads), and so do the streams of the others.
  const long long most = ((1ll << 32) - 1) / (64 * plan.waves);            // workgroups of a launch
  const long long all = chained ? plan.tiles : r.B, per = std::min(all, most / ((long long)plan.strips * (chained ? r.B : 1)));
  const size_t e = dtype == 1 ? 2 : 4, chunks = ((size_t)r.T + RC_KEEP - 1) / RC_KEEP;
  for (long long at = 0; at < all; at += per) {
    RecurrenceParams q = p;
    const long long n = std::min(per, all - at);
    if (!chained) {
      q.B = (int)n;
      const size_t row = (size_t)at * r.T, state = (size_t)at * r.D;
      auto rows = [&](auto*& of, size_t ld) { if (of) of = (char*)of + row * ld * e; };
      auto states = [&](auto*& of, size_t apart) { if (of) of += apart; };
      rows(q.z, q.ldz); rows(q.x, q.ldx); rows(q.dh, q.lddh); rows(q.h, q.ldh); rows(q.dz, q.lddz); rows(q.dx, q.lddx);
      states(q.h0, state); states(q.hT, state); states(q.dhT, state); states(q.dh0, state); states(q.states, state * chunks); states(q.lens, at);
    }
    const unsigned blocks = (unsigned)(n * plan.strips * (chained ? r.B : 1));
    if (dtype == 1) r.D >= RC_P ? rc_launch<bf16_t, true>(s, blocks, plan, q, backward) : rc_launch<bf16_t, false>(s, blocks, plan, q, backward);
    else r.D >= RC_P ? rc_launch<float, true>(s, blocks, plan, q, backward) : rc_launch<float, false>(s, blocks, plan, q, backward);
    const hipError_t err = hipGetLastError();
    if (err != hipSuccess) return err;
  }
  return hipSuccess;
}

}  // namespace ouro
