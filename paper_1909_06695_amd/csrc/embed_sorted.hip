// Gradient of the embedding lookup with a fixed order of summation (Eq. 7, left): dV[v, :] = scale * sum of the rows dh[n, :]
// with tok[n] = v.
//
// One launch, no workspace, no atomics on memory.  A workgroup owns the matrix rows v with v mod R = r and 128 bytes of
// columns of dh.  It reads all N ids (they stay in L2), keeps those of its rows as a list in LDS, sorts the list by row with a
// stable sort, and its teams of 8 lanes (16 bytes each) sum equal pieces of the sorted list: a frequent token is summed by
// many teams, whose parts are joined in order through LDS.  Every sum therefore has an order that only the ids determine.
// Rows are dealt to workgroups by v mod R because ids are usually ranked by frequency: neighbours are alike in weight.
//
// Bound by memory: N d elements read, the matrix written (or the rows of tokens that occur read and written).
#include "common.h"
#include "unaligned.h"

#include <algorithm>

namespace ouro {

constexpr int ES_THREADS = 512, ES_WAVES = ES_THREADS / 64;
constexpr int ES_TEAMS = ES_THREADS / STRIP_LANES;         // a team is the lanes of a strip: 128 bytes of a row of dh
constexpr int ES_STEP = 256;                               // ids of a wave at a time, four neighbours a lane
constexpr int ES_WAVE_CAP = 3 * ES_STEP, ES_CAP = ES_WAVES * ES_WAVE_CAP;     // entries of the list, of which each wave fills its part
constexpr int ES_RANK = ES_THREADS;                        // longest list that is sorted by counting smaller entries
constexpr int ES_BITS = 9, ES_BINS = 1 << ES_BITS;         // largest digit of the radix sort
constexpr int ES_ROW_BITS = 14;                            // matrix rows of a workgroup: a bit each, two digits
constexpr int ES_CLEARERS = 256;                           // workgroups that clear rows, one a CU
static_assert(ES_BINS == ES_THREADS, "one bin a thread");

struct EmbedSortedParams {
  const int32_t* tok; const void* dh; float* dV;
  size_t lddh, ldv;
  int N, d, vocab;
  int slices, log2R;
  int clearers, zero_rows;                                 // the first workgroups clear zero_rows rows each; 0: the sums are added
  int n_bits, row_bits;                                    // an entry is (matrix row of the workgroup) << n_bits | position in ids
  float scale;
};

// Four neighbouring ids, -1 behind the end.
__device__ __forceinline__ int4 es_ids(const EmbedSortedParams& p, int at) {
  int v[4] = {-1, -1, -1, -1};
  if (at + 4 <= p.N) load_unaligned<int32_t, 4>(p.tok + at, v);
  else if (at < p.N) {
    v[0] = p.tok[at];
    if (at + 1 < p.N) v[1] = p.tok[at + 1];
    if (at + 2 < p.N) v[2] = p.tok[at + 2];
  }
  return make_int4(v[0], v[1], v[2], v[3]);
}

// Lanes of the wave whose `key` (bits wide) equals this lane's, among those of `in`.
__device__ __forceinline__ uint64_t es_peers(uint32_t key, int bits, uint64_t in) {
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((key >> b) & 1);
    in &= (key >> b) & 1 ? set : ~set;
  }
  return in;
}

// Clears the rows [z0, z1) without a token: neighbouring rows, whole, so that full cache lines are written.
__device__ __forceinline__ void es_clear(const EmbedSortedParams& p, uint32_t z0, uint32_t z1, uint32_t* touched) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (uint32_t i = tid; i < (z1 - z0 + 31) / 32; i += ES_THREADS) touched[i] = 0;
  __syncthreads();
#pragma unroll 2
  for (int n = 4 * tid; n < p.N; n += 4 * ES_THREADS) {
    const int4 v = es_ids(p, n);
    auto mark = [&](int id) __attribute__((always_inline)) {
      const uint32_t r = (uint32_t)id - z0;
      if (id >= 0 && r < z1 - z0) atomicOr(&touched[r >> 5], 1u << (r & 31));
    };
    mark(v.x); mark(v.y); mark(v.z); mark(v.w);
  }
  __syncthreads();
  int lanes = 1;                                           // of a row, 16 bytes each
  while (lanes < 64 && lanes * 4 < p.d) lanes *= 2;
  const int rows = 64 / lanes, c0 = lane % lanes * 4;
  const float zero[4] = {};
  for (uint32_t i = wave * rows + lane / lanes; i < z1 - z0; i += ES_WAVES * rows) {
    if (touched[i >> 5] >> (i & 31) & 1) continue;
    float* out = p.dV + (z0 + i) * p.ldv;
    for (int c = c0; c < p.d; c += lanes * 4) {
      if (c + 4 <= p.d) store_unaligned<float, 4>(out + c, zero);
      else
        for (int e = c; e < p.d; ++e) out[e] = 0.f;
    }
  }
}

// WHOLE: see lane_columns.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(ES_THREADS, 4) void embed_bwd_sorted_kernel(EmbedSortedParams p) {
  constexpr int P = 16 / sizeof(T);                        // columns of a lane
  constexpr int W = STRIP_LANES * P;                       // columns of the workgroup
  __shared__ __align__(16) uint32_t list_a[ES_CAP], list_b[ES_CAP];
  __shared__ __align__(16) uint32_t hist_or_heads[ES_WAVES * ES_BINS];
  __shared__ uint32_t seen[1 << (ES_ROW_BITS - 5)];
  __shared__ uint32_t count[ES_WAVES], bins[ES_WAVES];
  __shared__ uint8_t through[ES_WAVES];
  static_assert(ES_TEAMS * W <= ES_WAVES * ES_BINS, "the heads fit the histogram's place");
  if ((int)blockIdx.x < p.clearers) {
    const uint32_t z0 = (uint32_t)min((uint64_t)blockIdx.x * p.zero_rows, (uint64_t)p.vocab), z1 = (uint32_t)min((uint64_t)z0 + p.zero_rows, (uint64_t)p.vocab);
    es_clear(p, z0, z1, list_a);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  int4 next = es_ids(p, wave * ES_STEP + 4 * lane);
  const uint32_t block = blockIdx.x - p.clearers, R = 1u << p.log2R, mine = block / p.slices;
  const LaneColumns own = lane_columns<P, WHOLE>(block % p.slices, lane % STRIP_LANES, p.d);
  const int team = tid / STRIP_LANES;
  const uint64_t below = (1ull << lane) - 1;
  const bool overwrite = p.clearers > 0;
  for (int i = tid; i < 1 << max(0, p.row_bits - 5); i += ES_THREADS) seen[i] = 0;

  bool first = true, end = false;
  int n0 = 0;                                              // ids before n0 have been looked at
  while (!end) {
    // ---- the entries among the ids, in order for each wave
    const int n_base = n0;
    int k = 0;
    for (int steps = 0;; ++steps) {
      end = n0 >= p.N;
      if (end || n0 - n_base > (1 << p.n_bits) - ES_WAVES * ES_STEP) break;
      if (steps >= ES_WAVE_CAP / ES_STEP && __syncthreads_or(k > ES_WAVE_CAP - ES_STEP)) break;
      const int4 v = next;
      const int at = n0 + wave * ES_STEP + 4 * lane;
      next = es_ids(p, at + ES_WAVES * ES_STEP);
      auto take = [&](uint32_t id, int n) __attribute__((always_inline)) {
        const bool on = id < (uint32_t)p.vocab && (id & (R - 1)) == mine;
        const uint64_t all = __ballot(on);
        if (on) list_a[wave * ES_WAVE_CAP + k + (int)__popcll(all & below)] = id >> p.log2R << p.n_bits | (uint32_t)n;
        k += (int)__popcll(all);
      };
      take(v.x, at - n_base); take(v.y, at + 1 - n_base); take(v.z, at + 2 - n_base); take(v.w, at + 3 - n_base);
      n0 += ES_WAVES * ES_STEP;
    }
    if (lane == 0) count[wave] = (uint32_t)k;
    __syncthreads();
    int m = 0, at = 0;
#pragma unroll
    for (int w = 0; w < ES_WAVES; ++w) {
      at += w < wave ? (int)count[w] : 0;
      m += (int)count[w];
    }
    for (int i = lane; i < k; i += 64) list_b[at + i] = list_a[wave * ES_WAVE_CAP + i];
    __syncthreads();
    // ---- a stable sort by row
    const uint32_t* key = list_b;
    if (m > 1 && m <= ES_RANK) {
      if (tid < m) {                                       // entries differ: the place of one is the number of smaller ones
        const uint32_t e = list_b[tid];
        uint32_t rank = 0;
        int j = 0;
#pragma unroll 4
        for (; j + 4 <= m; j += 4) {
          const uint4 o = *reinterpret_cast<const uint4*>(list_b + j);
          rank += (uint32_t)(o.x < e) + (uint32_t)(o.y < e) + (uint32_t)(o.z < e) + (uint32_t)(o.w < e);
        }
        for (; j < m; ++j) rank += (uint32_t)(list_b[j] < e);
        list_a[rank] = e;
      }
      key = list_a;
      __syncthreads();
    } else if (m > ES_RANK) {
      uint32_t* hist = hist_or_heads + wave * ES_BINS;     // [wave][bin]
      const int per = (m + ES_THREADS - 1) / ES_THREADS * 64, e0 = min(m, wave * per), e1 = min(m, e0 + per);
      uint32_t *from = list_b, *to = list_a;
      const int passes = (max(1, p.row_bits) + ES_BITS - 1) / ES_BITS, digit = (max(1, p.row_bits) + passes - 1) / passes;
      for (int shift = p.n_bits; shift < p.n_bits + max(1, p.row_bits); shift += digit) {
        const uint32_t mask = (1u << digit) - 1;
        for (int i = lane; i < ES_BINS / 4; i += 64) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
        for (int i = e0; i < e1; i += 64) {                // how many a bin
          const bool on = i + lane < e1;
          const uint32_t bin = on ? (from[i + lane] >> shift) & mask : 0;
          const uint64_t peers = es_peers(bin, digit, __ballot(on));
          if (on && !(peers & below)) hist[bin] += (uint32_t)__popcll(peers);
          __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        uint32_t sum = 0;                                  // this thread's bin over the waves, then over the bins before
#pragma unroll
        for (int w = 0; w < ES_WAVES; ++w) sum += hist_or_heads[w * ES_BINS + tid];
        uint32_t incl = sum;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
          const uint32_t y = __shfl_up(incl, o, 64);
          if (lane >= o) incl += y;
        }
        if (lane == 63) bins[wave] = incl;
        __syncthreads();
        uint32_t base = incl - sum;
#pragma unroll
        for (int w = 0; w < ES_WAVES; ++w) base += w < wave ? bins[w] : 0;
#pragma unroll
        for (int w = 0; w < ES_WAVES; ++w) {
          const uint32_t had = hist_or_heads[w * ES_BINS + tid];
          hist_or_heads[w * ES_BINS + tid] = base;
          base += had;
        }
        __syncthreads();
        for (int i = e0; i < e1; i += 64) {                // where each goes
          const bool on = i + lane < e1;
          const uint32_t e = on ? from[i + lane] : 0, bin = (e >> shift) & mask;
          const uint64_t peers = es_peers(bin, digit, __ballot(on));
          uint32_t place = 0;
          if (on) {
            place = hist[bin];
            to[place + (uint32_t)__popcll(peers & below)] = e;
          }
          __builtin_amdgcn_wave_barrier();
          if (on && !(peers & below)) hist[bin] = place + (uint32_t)__popcll(peers);
          __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        uint32_t* t = from; from = to; to = t;
      }
      key = from;
    }
    // ---- sums: a team takes an equal piece of the sorted list
    float* heads = reinterpret_cast<float*>(hist_or_heads);    // [team][W]: a team's part of a sum that an earlier team owns
    const int per = (m + ES_TEAMS - 1) / ES_TEAMS, s = min(m, team * per), e = min(m, s + per);
    const uint32_t mask_n = (1u << p.n_bits) - 1;
    float acc[P] = {}, old[P] = {};                        // of the sum under way; what the matrix holds
    auto place = [&](uint32_t r) __attribute__((always_inline)) { return p.dV + ((size_t)r << p.log2R | mine) * p.ldv + own.col; };
    auto write = [&](uint32_t r) __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < P; ++j) old[j] = fmaf(p.scale, acc[j], old[j]);
      store_columns<float, P, WHOLE>(place(r), old, own.n);
    };
    bool pending = false, middle = false;                  // the last sum goes on in the next team's piece, and began here or before
    uint32_t cur = 0;
    if (s < e) {
      const T* dh = reinterpret_cast<const T*>(p.dh) + n_base * p.lddh + own.col;
      cur = key[s] >> p.n_bits;
      bool head = s > 0 && key[s - 1] >> p.n_bits == cur;
      uint32_t before = head ? cur : ~0u;                  // row of the entry before the ones requested
      constexpr int U = 4;                                 // rows requested together, with the matrix rows of sums that begin
      for (int i = s; i < e; i += U) {
        UnalignedPack<T, P> x[U] = {};
        UnalignedPack<float, P> had[U] = {};
        uint32_t r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t entry = key[min(i + u, e - 1)];
          r[u] = entry >> p.n_bits;
          if (i + u < e) {
            load_raw_columns<T, P, WHOLE>(dh + (size_t)(entry & mask_n) * p.lddh, x[u], own.n);
            if (r[u] != before && (!overwrite || (!first && (seen[r[u] >> 5] >> (r[u] & 31) & 1)))) load_raw_columns<float, P, WHOLE>(place(r[u]), had[u], own.n);
          }
          before = r[u];
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i + u < e) {
            const bool change = r[u] != cur;
            if (change) {
              if (head) {
#pragma unroll
                for (int j = 0; j < P; ++j) heads[team * W + (lane % STRIP_LANES) * P + j] = acc[j];
              } else {
                write(cur);
              }
              head = false;
              cur = r[u];
            }
            if (change || (i + u == s && !head)) {
#pragma unroll
              for (int j = 0; j < P; ++j) { acc[j] = 0.f; old[j] = had[u].v[j]; }
            }
#pragma unroll
            for (int j = 0; j < P; ++j) acc[j] += to_f32(x[u].v[j]);
          }
      }
      const bool goes_on = e < m && key[e] >> p.n_bits == cur;
      pending = goes_on && !head;
      middle = goes_on && head;
      if (head) {
#pragma unroll
        for (int j = 0; j < P; ++j) heads[team * W + (lane % STRIP_LANES) * P + j] = acc[j];
      } else if (!pending) {
        write(cur);
      }
    }
    const uint64_t middles = __ballot(middle);             // one bit a team
    if (lane == 0) {
      uint32_t bits = 0;
      for (int t = 0; t < 64 / STRIP_LANES; ++t) bits |= (uint32_t)(middles >> (t * STRIP_LANES) & 1) << t;
      through[wave] = (uint8_t)bits;
    }
    __syncthreads();
    if (pending) {
      uint64_t mask = 0;
#pragma unroll
      for (int w = 0; w < ES_WAVES; ++w) mask |= (uint64_t)through[w] << (w * 8);
      const int more = (int)__ffsll((unsigned long long)~(mask >> team >> 1));    // teams that hold the rest
      const float* h = heads + (team + 1) * W + (lane % STRIP_LANES) * P;
#pragma unroll 4
      for (int t = 0; t < more; ++t)
#pragma unroll
        for (int j = 0; j < P; ++j) acc[j] += h[t * W + j];
      write(cur);
    }
    if (!end) {
      __syncthreads();
      for (int i = tid; i < m; i += ES_THREADS) atomicOr(&seen[key[i] >> p.n_bits >> 5], 1u << (key[i] >> p.n_bits & 31));
      __syncthreads();
    }
    first = false;
  }
}

hipError_t launch_embed_bwd_sorted(hipStream_t s, int dtype, const int32_t* tok, const void* dh, int lddh, float* dV, int ldv, int N, int d,
                                   int vocab, float scale, int accumulate) {
  EmbedSortedParams p;
  memset(&p, 0, sizeof p);
  p.tok = tok; p.dh = dh; p.dV = dV; p.lddh = lddh; p.ldv = ldv; p.N = N; p.d = d; p.vocab = vocab; p.scale = scale;
  p.slices = dtype == 1 ? strip_count<8>(d) : strip_count<4>(d);
  // As many workgroups as the chip holds at once, two a CU, of which half clear rows where the matrix is overwritten; four
  // matrix rows each at least, and as many workgroups as keep the bit maps within their sizes.
  p.clearers = accumulate ? 0 : std::min((vocab + 3) / 4, std::max(ES_CLEARERS, (int)((vocab + 32ll * ES_CAP - 1) / (32ll * ES_CAP))));
  p.zero_rows = accumulate ? 0 : (vocab + p.clearers - 1) / p.clearers;
  while (((long long)p.slices << (p.log2R + 1)) <= (accumulate ? 512 : 256) && (4ll << p.log2R) < vocab) ++p.log2R;
  while ((1ll << ES_ROW_BITS << p.log2R) < vocab) ++p.log2R;
  while ((1ll << p.row_bits << p.log2R) < vocab) ++p.row_bits;
  p.n_bits = std::min(30, 32 - p.row_bits);
  const long long blocks = ((long long)p.slices << p.log2R) + p.clearers;
  if (blocks * ES_THREADS >> 32) return hipErrorInvalidValue;
  dim3 grid((unsigned)blocks), block(ES_THREADS);
  if (dtype == 1) {
    if (d >= 8) hipLaunchKernelGGL((embed_bwd_sorted_kernel<bf16_t, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((embed_bwd_sorted_kernel<bf16_t, false>), grid, block, 0, s, p);
  } else {
    if (d >= 4) hipLaunchKernelGGL((embed_bwd_sorted_kernel<float, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((embed_bwd_sorted_kernel<float, false>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace ouro
