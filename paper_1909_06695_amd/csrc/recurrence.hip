// Gated linear recurrence h_t = f_t h_{t-1} + (1 - f_t) x_t, f_t = sigmoid(z_t), forward and backward.
//
// A step is the affine map h -> f h + u with u = (1 - f) x, and maps compose: (A, H) after (a, h) is (A a, A h + H).  So a thread
// takes a few consecutive steps of a few channels and composes their maps, the rows of a wave and then the waves of a
// workgroup scan over these, and with the state that enters its steps known each thread runs them once more from registers.
// Backward, with G_t = dh_t + f_{t+1} G_{t+1} and P_t = f_t G_t: P_t = f_t P_{t+1} + f_t dh_t, the same kind of map from the right with the
// same factors; dx_t = (1 - f_t) G_t, dz_t = G_t (h_{t-1} - x_t) f_t (1 - f_t).  h is formed again from the fp32 states that the forward
// pass left at every 64th step, so that it is neither read back nor rounded.
//
// Bound by memory: z, x (and dh) read, h (or dz, dx) written.  A workgroup owns 128 bytes of channels of one stream, a tile
// of steps at a time.  Few streams and channels leave the chip empty: the steps are then cut into segments, a first launch
// leaves the maps of whole segments in the workspace and the second starts each segment from their composition; it costs
// a second reading of z and x (z and dh).
#include "common.h"
#include "unaligned.h"

#include <algorithm>

namespace ouro {

constexpr int RC_LANES = STRIP_LANES, RC_ROWS = 64 / RC_LANES;       // of a wave: 8 rows of 8 lanes, 16 bytes a lane
constexpr int RC_WAVES = 8;                                // most waves of a workgroup
template <typename T> struct RcShape {
  static constexpr int P = 16 / sizeof(T);                 // channels of a lane
  static constexpr int L = 32 / P;                         // consecutive steps of a lane: 32 elements in registers
  static constexpr int W = RC_LANES * P;                   // channels of a workgroup
  static constexpr int STEPS = RC_ROWS * L;                // steps of a wave
};
constexpr int RC_KEEP = RECURRENCE_STRIDE;
static_assert(RC_KEEP % RcShape<float>::STEPS == 0 && RC_KEEP % RcShape<bf16_t>::STEPS == 0, "a kept state every whole number of waves");

struct RecurrenceParams {
  int B, T, D, strips, segs, seg_steps;
  const void* z; const void* x; const void* dh;
  size_t ldz, ldx, lddh;
  const float* h0; const float* dhT; const int32_t* lens;
  void* h; void* dz; void* dx;
  size_t ldh, lddz, lddx;
  float* hT; float* dh0; float* states;
  float* maps;                                             // [B][segs][2][D]: factor and offset of whole segments
};

// f and 1 - f from one exponential, neither by subtraction; z = +-infinity gives exactly 1 and 0.
__device__ __forceinline__ void rc_gate(float z, float& f, float& e) {
  const float t = __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(z)), r = __builtin_amdgcn_rcpf(1.f + t), q = t * r;
  f = z >= 0.f ? r : q;
  e = z >= 0.f ? q : r;
  if (z != z) f = e = z;
}

// What a thread needs to find its elements.
struct RcPlace {
  int b, seg, col, ncol, wave, row, lane8, waves, t0, t1, len;     // t0, t1: the segment's steps
  size_t base;                                             // row of step 0
};
template <typename T, bool WHOLE>
__device__ __forceinline__ RcPlace rc_place(const RecurrenceParams& p) {
  RcPlace a;
  const int strip = blockIdx.x % p.strips, rest = blockIdx.x / p.strips;
  a.seg = rest % p.segs;
  a.b = rest / p.segs;
  a.lane8 = threadIdx.x & (RC_LANES - 1);
  a.row = (threadIdx.x & 63) / RC_LANES;
  a.wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  a.waves = blockDim.x >> 6;
  const LaneColumns own = lane_columns<RcShape<T>::P, WHOLE>(strip, a.lane8, p.D);
  a.col = own.col;
  a.ncol = own.n;
  a.t0 = a.seg * p.seg_steps;
  a.t1 = min(p.T, a.t0 + p.seg_steps);
  a.len = p.lens ? max(0, min(p.T, p.lens[a.b])) : p.T;
  a.base = (size_t)a.b * p.T;
  return a;
}

// The exclusive scan of (A, H) over the rows of a wave; the last row's inclusive value goes to LDS.  UP: rows below come first.
template <int P, bool UP>
__device__ __forceinline__ void rc_wave_scan(const RcPlace& a, float (&A)[P], float (&H)[P], float* sA, float* sH) {
#pragma unroll
  for (int o = 1; o < RC_ROWS; o <<= 1) {
    const bool on = UP ? a.row >= o : a.row + o < RC_ROWS;
#pragma unroll
    for (int j = 0; j < P; ++j) {
      const float pa = UP ? __shfl_up(A[j], o * RC_LANES, 64) : __shfl_down(A[j], o * RC_LANES, 64);
      const float ph = UP ? __shfl_up(H[j], o * RC_LANES, 64) : __shfl_down(H[j], o * RC_LANES, 64);
      if (on) { H[j] = fmaf(A[j], ph, H[j]); A[j] *= pa; }
    }
  }
  if (a.row == (UP ? RC_ROWS - 1 : 0)) {
#pragma unroll
    for (int j = 0; j < P; ++j) { if (sA) sA[j] = A[j]; sH[j] = H[j]; }
  }
#pragma unroll
  for (int j = 0; j < P; ++j) {
    const float pa = UP ? __shfl_up(A[j], RC_LANES, 64) : __shfl_down(A[j], RC_LANES, 64);
    const float ph = UP ? __shfl_up(H[j], RC_LANES, 64) : __shfl_down(H[j], RC_LANES, 64);
    const bool on = UP ? a.row > 0 : a.row + 1 < RC_ROWS;
    A[j] = on ? pa : 1.f;
    H[j] = on ? ph : 0.f;
  }
}

// The map of a segment in the workspace.  That of the first one (in the direction of the scan) holds instead of its factor the
// state that enters it and instead of its offset the state behind it: h0 and hT may be one buffer, and the second launch, in which
// segments run in any order, would read the one and write the other.
__device__ __forceinline__ float* rc_map(const RecurrenceParams& p, const RcPlace& a, int seg) {
  return p.maps + ((size_t)a.b * p.segs + seg) * 2 * p.D + a.col;
}
// state <- what enters the segment.  UP: segments before it come first; `from` is h0 or dhT.
template <int P, bool WHOLE, bool UP, bool MAPS>
__device__ __forceinline__ void rc_enter(const RecurrenceParams& p, const RcPlace& a, const float* from, float (&state)[P]) {
  const int first = UP ? 0 : p.segs - 1, step = UP ? 1 : -1;
  if (MAPS || p.segs == 1) {
    if (a.seg == first && from) load_columns<float, P, WHOLE>(from + (size_t)a.b * p.D + a.col, state, a.ncol);
    return;
  }
  if (a.seg == first) {
    load_columns<float, P, WHOLE>(rc_map(p, a, first), state, a.ncol);
    return;
  }
  load_columns<float, P, WHOLE>(rc_map(p, a, first) + p.D, state, a.ncol);
#pragma unroll 4
  for (int s = first + step; s != a.seg; s += step) {
    float A[P] = {}, H[P] = {};
    load_columns<float, P, WHOLE>(rc_map(p, a, s), A, a.ncol);
    load_columns<float, P, WHOLE>(rc_map(p, a, s) + p.D, H, a.ncol);
#pragma unroll
    for (int j = 0; j < P; ++j) state[j] = fmaf(A[j], state[j], H[j]);
  }
}
template <int P, bool WHOLE, bool UP>
__device__ __forceinline__ void rc_leave_map(const RecurrenceParams& p, const RcPlace& a, const float* from, const float (&factor)[P], const float (&state)[P]) {
  float in[P] = {};
  const bool first = a.seg == (UP ? 0 : p.segs - 1);
  if (first) rc_enter<P, WHOLE, UP, true>(p, a, from, in);
#pragma unroll
  for (int j = 0; j < P; ++j) in[j] = first ? in[j] : factor[j];
  store_columns<float, P, WHOLE>(rc_map(p, a, a.seg), in, a.ncol);
  store_columns<float, P, WHOLE>(rc_map(p, a, a.seg) + p.D, state, a.ncol);
}

// MAPS: only the map of the segment.  WHOLE: see lane_columns.
template <typename T, bool WHOLE, bool MAPS>
__global__ __launch_bounds__(64 * RC_WAVES) void recurrence_fwd_kernel(RecurrenceParams p) {
  constexpr int P = RcShape<T>::P, L = RcShape<T>::L, W = RcShape<T>::W, STEPS = RcShape<T>::STEPS;
  __shared__ float sA[2][RC_WAVES][W], sH[2][RC_WAVES][W];
  const RcPlace a = rc_place<T, WHOLE>(p);
  if (MAPS && a.seg == p.segs - 1) return;                 // nothing starts behind the last segment
  const T* z = reinterpret_cast<const T*>(p.z) + a.col;
  const T* x = reinterpret_cast<const T*>(p.x) + a.col;
  float state[P] = {}, factor[P];
#pragma unroll
  for (int j = 0; j < P; ++j) factor[j] = 1.f;
  rc_enter<P, WHOLE, true, MAPS>(p, a, p.h0, state);
  int buf = 0;
  for (int tile = a.t0; tile < a.t1; tile += a.waves * STEPS, buf ^= 1) {
    const int t = tile + a.wave * STEPS + a.row * L;
    float f[L][P] = {}, u[L][P] = {};
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (t + i < min(a.t1, a.len)) {
        load_columns<T, P, WHOLE>(z + (a.base + t + i) * p.ldz, f[i], a.ncol);
        load_columns<T, P, WHOLE>(x + (a.base + t + i) * p.ldx, u[i], a.ncol);
      }
    }
    float A[P], H[P];
#pragma unroll
    for (int j = 0; j < P; ++j) { A[j] = 1.f; H[j] = 0.f; }
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const bool live = t + i < min(a.t1, a.len);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        if (live) {
          float e;
          rc_gate(f[i][j], f[i][j], e);
          u[i][j] *= e;
        } else { f[i][j] = 1.f; u[i][j] = 0.f; }           // a step that is not taken keeps the state
        A[j] *= f[i][j];
        H[j] = fmaf(f[i][j], H[j], u[i][j]);
      }
    }
    rc_wave_scan<P, true>(a, A, H, &sA[buf][a.wave][a.lane8 * P], &sH[buf][a.wave][a.lane8 * P]);
    __syncthreads();
    float in[P];
    for (int w = 0; w < a.waves; ++w) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        if (w == a.wave) in[j] = state[j];
        state[j] = fmaf(sA[buf][w][a.lane8 * P + j], state[j], sH[buf][w][a.lane8 * P + j]);
        if (MAPS) factor[j] *= sA[buf][w][a.lane8 * P + j];
      }
    }
    if (MAPS) continue;
    float h[P];
#pragma unroll
    for (int j = 0; j < P; ++j) h[j] = fmaf(A[j], in[j], H[j]);
    if (p.states && t % RC_KEEP == 0 && t < a.t1)
      store_columns<float, P, WHOLE>(p.states + ((size_t)a.b * ((p.T + RC_KEEP - 1) / RC_KEEP) + t / RC_KEEP) * p.D + a.col, h, a.ncol);
#pragma unroll
    for (int i = 0; i < L; ++i) {
      float out[P];
#pragma unroll
      for (int j = 0; j < P; ++j) {
        h[j] = fmaf(f[i][j], h[j], u[i][j]);
        out[j] = t + i < a.len ? h[j] : 0.f;
      }
      if (t + i < a.t1) store_columns<T, P, WHOLE>(reinterpret_cast<T*>(p.h) + (a.base + t + i) * p.ldh + a.col, out, a.ncol);
    }
  }
  if (a.wave == 0 && a.row == 0) {
    if (MAPS) {
      rc_leave_map<P, WHOLE, true>(p, a, p.h0, factor, state);
    } else if (a.seg == p.segs - 1 && p.hT) {
      store_columns<float, P, WHOLE>(p.hT + (size_t)a.b * p.D + a.col, state, a.ncol);
    }
  }
}

template <typename T, bool WHOLE, bool MAPS>
__global__ __launch_bounds__(64 * RC_WAVES) void recurrence_bwd_kernel(RecurrenceParams p) {
  constexpr int P = RcShape<T>::P, L = RcShape<T>::L, W = RcShape<T>::W, STEPS = RcShape<T>::STEPS;
  __shared__ float sA[2][RC_WAVES][W], sH[2][RC_WAVES][W], sQ[2][RC_WAVES][W];
  const RcPlace a = rc_place<T, WHOLE>(p);
  if (MAPS && a.seg == 0) return;                          // nothing starts before the first segment
  const T* z = reinterpret_cast<const T*>(p.z) + a.col;
  const T* x = reinterpret_cast<const T*>(p.x) + a.col;
  const T* g = reinterpret_cast<const T*>(p.dh) + a.col;
  float state[P] = {}, factor[P];                          // P of the step behind the tile
#pragma unroll
  for (int j = 0; j < P; ++j) factor[j] = 1.f;
  rc_enter<P, WHOLE, false, MAPS>(p, a, p.dhT, state);
  const int steps = a.waves * STEPS;
  int buf = 0;
  for (int tile = a.t0 + (a.t1 - a.t0 - 1) / steps * steps; tile >= a.t0; tile -= steps, buf ^= 1) {
    const int tw = tile + a.wave * STEPS, t = tw + a.row * L;
    float f[L][P] = {}, e[L][P], v[L][P] = {}, G[L][P] = {}, kept[P] = {};
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (t + i < min(a.t1, a.len)) {
        load_columns<T, P, WHOLE>(z + (a.base + t + i) * p.ldz, f[i], a.ncol);
        load_columns<T, P, WHOLE>(g + (a.base + t + i) * p.lddh, G[i], a.ncol);
        if (!MAPS) load_columns<T, P, WHOLE>(x + (a.base + t + i) * p.ldx, v[i], a.ncol);
      }
    }
    if (!MAPS && tw < a.t1) load_columns<float, P, WHOLE>(p.states + ((size_t)a.b * ((p.T + RC_KEEP - 1) / RC_KEEP) + tw / RC_KEEP) * p.D + a.col, kept, a.ncol);
    float A[P], H[P], B[P], Q[P];
#pragma unroll
    for (int j = 0; j < P; ++j) { A[j] = 1.f; H[j] = Q[j] = 0.f; }
#pragma unroll
    for (int i = 0; i < L; ++i) {
      const bool live = t + i < min(a.t1, a.len);
#pragma unroll
      for (int j = 0; j < P; ++j) {
        if (live) {
          rc_gate(f[i][j], f[i][j], e[i][j]);
        } else { f[i][j] = 1.f; e[i][j] = v[i][j] = G[i][j] = 0.f; }
        A[j] *= f[i][j];
        if (!MAPS) H[j] = fmaf(f[i][j], H[j], e[i][j] * v[i][j]);
      }
    }
#pragma unroll
    for (int i = L - 1; i >= 0; --i)
#pragma unroll
      for (int j = 0; j < P; ++j) Q[j] = f[i][j] * (G[i][j] + Q[j]);
#pragma unroll
    for (int j = 0; j < P; ++j) B[j] = A[j];
    rc_wave_scan<P, false>(a, B, Q, &sA[buf][a.wave][a.lane8 * P], &sQ[buf][a.wave][a.lane8 * P]);
    if (!MAPS) rc_wave_scan<P, true>(a, A, H, nullptr, &sH[buf][a.wave][a.lane8 * P]);
    __syncthreads();
    float in[P];
    for (int w = a.waves - 1; w >= 0; --w) {
#pragma unroll
      for (int j = 0; j < P; ++j) {
        if (w == a.wave) in[j] = state[j];
        state[j] = fmaf(sA[buf][w][a.lane8 * P + j], state[j], sQ[buf][w][a.lane8 * P + j]);
        if (MAPS) factor[j] *= sA[buf][w][a.lane8 * P + j];
      }
    }
    if (MAPS) continue;
    // the state that enters the wave: kept, or one or more waves behind a kept one
    for (int w = a.wave - (tw % RC_KEEP) / STEPS; w < a.wave; ++w)
#pragma unroll
      for (int j = 0; j < P; ++j) kept[j] = fmaf(sA[buf][w][a.lane8 * P + j], kept[j], sH[buf][w][a.lane8 * P + j]);
#pragma unroll
    for (int j = 0; j < P; ++j) {
      float h = fmaf(A[j], kept[j], H[j]);
#pragma unroll
      for (int i = 0; i < L; ++i) {
        const float u = e[i][j] * v[i][j];
        v[i][j] = h - v[i][j];
        h = fmaf(f[i][j], h, u);
      }
      float q = fmaf(B[j], in[j], Q[j]);
#pragma unroll
      for (int i = L - 1; i >= 0; --i) {
        G[i][j] += q;
        q = f[i][j] * G[i][j];
      }
    }
#pragma unroll
    for (int i = 0; i < L; ++i) {
      if (t + i >= a.t1) continue;
      float dx[P], dz[P];
#pragma unroll
      for (int j = 0; j < P; ++j) {
        const bool live = t + i < a.len;
        dx[j] = live ? e[i][j] * G[i][j] : 0.f;
        dz[j] = live ? G[i][j] * v[i][j] * (f[i][j] * e[i][j]) : 0.f;
      }
      store_columns<T, P, WHOLE>(reinterpret_cast<T*>(p.dx) + (a.base + t + i) * p.lddx + a.col, dx, a.ncol);
      store_columns<T, P, WHOLE>(reinterpret_cast<T*>(p.dz) + (a.base + t + i) * p.lddz + a.col, dz, a.ncol);
    }
  }
  if (a.wave == 0 && a.row == 0) {
    if (MAPS) {
      rc_leave_map<P, WHOLE, false>(p, a, p.dhT, factor, state);
    } else if (a.seg == 0 && p.dh0) {
      store_columns<float, P, WHOLE>(p.dh0 + (size_t)a.b * p.D + a.col, state, a.ncol);
    }
  }
}

// How a call is laid out: waves of a workgroup and segments.
struct RcPlan { int strips, waves, segs, seg_steps; };
static RcPlan rc_plan(int dtype, int B, int T, int D) {
  RcPlan r;
  const int steps = dtype == 1 ? RcShape<bf16_t>::STEPS : RcShape<float>::STEPS;
  r.strips = dtype == 1 ? strip_count<8>(D) : strip_count<4>(D);
  r.waves = 1;
  while (r.waves < RC_WAVES && (long long)r.waves * steps < T) r.waves *= 2;
  const int tile = r.waves * steps, tiles = (int)(((long long)T + tile - 1) / tile);
  const long long blocks = (long long)B * r.strips;
  r.segs = (int)std::min<long long>(std::min(tiles, 64), (512 + blocks - 1) / blocks);
  const int per = (tiles + r.segs - 1) / r.segs;
  r.seg_steps = per * tile;
  r.segs = (tiles + per - 1) / per;
  return r;
}
size_t recurrence_scratch_floats(int B, int T, int D) {
  size_t n = 0;
  for (int dtype = 0; dtype < 2; ++dtype) {
    const RcPlan r = rc_plan(dtype, B, T, D);
    if (r.segs > 1) n = std::max(n, (size_t)B * r.segs * 2 * D);
  }
  return n;
}

template <typename T, bool WHOLE, bool MAPS>
static void rc_launch(hipStream_t s, unsigned blocks, int waves, const RecurrenceParams& p, bool backward) {
  if (backward) hipLaunchKernelGGL((recurrence_bwd_kernel<T, WHOLE, MAPS>), dim3(blocks), dim3(64 * waves), 0, s, p);
  else hipLaunchKernelGGL((recurrence_fwd_kernel<T, WHOLE, MAPS>), dim3(blocks), dim3(64 * waves), 0, s, p);
}
template <typename T, bool WHOLE>
static hipError_t rc_launch(hipStream_t s, unsigned blocks, int waves, const RecurrenceParams& p, bool backward) {
  if (p.segs > 1) {
    rc_launch<T, WHOLE, true>(s, blocks, waves, p, backward);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  rc_launch<T, WHOLE, false>(s, blocks, waves, p, backward);
  return hipGetLastError();
}
hipError_t launch_recurrence(hipStream_t s, int dtype, const RecurrenceDesc& r) {
  const RcPlan plan = rc_plan(dtype, r.B, r.T, r.D);
  const long long blocks = (long long)r.B * plan.strips * plan.segs;
  if (blocks * 64 * plan.waves >> 32 || (plan.segs > 1 && !r.scratch)) return hipErrorInvalidValue;
  RecurrenceParams p;
  memset(&p, 0, sizeof p);
  p.B = r.B; p.T = r.T; p.D = r.D; p.strips = plan.strips; p.segs = plan.segs; p.seg_steps = plan.seg_steps;
  p.z = r.z; p.x = r.x; p.dh = r.dh; p.ldz = r.ldz; p.ldx = r.ldx; p.lddh = r.lddh;
  p.h0 = r.h0; p.dhT = r.dhT; p.lens = r.lens;
  p.h = r.h; p.dz = r.dz; p.dx = r.dx; p.ldh = r.ldh; p.lddz = r.lddz; p.lddx = r.lddx;
  p.hT = r.hT; p.dh0 = r.dh0; p.states = r.states; p.maps = r.scratch;
  const bool backward = r.dz != nullptr;
  if (dtype == 1) return r.D >= 8 ? rc_launch<bf16_t, true>(s, (unsigned)blocks, plan.waves, p, backward) : rc_launch<bf16_t, false>(s, (unsigned)blocks, plan.waves, p, backward);
  return r.D >= 4 ? rc_launch<float, true>(s, (unsigned)blocks, plan.waves, p, backward) : rc_launch<float, false>(s, (unsigned)blocks, plan.waves, p, backward);
}

}  // namespace ouro
