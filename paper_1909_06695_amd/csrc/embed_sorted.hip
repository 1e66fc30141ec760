// Gradient of the embedding lookup with a fixed order of summation (Eq. 7, left): dV[v, :] = scale * sum of the rows dh[n, :]
// with tok[n] = v.
//
// One launch, no workspace, no atomics on memory.  A workgroup owns the matrix rows v with v mod R = r and 128 bytes of
// columns of dh.  It reads all N ids (they stay in L2), keeps those of its rows as a list in LDS, sorts the list by row with a
// stable sort, and its teams of 8 lanes (16 bytes each) sum equal pieces of the sorted list: a frequent token is summed by
// many teams, whose parts are joined in order through LDS; one of thousands of ids is summed without a list.  Every sum therefore
// has an order that only the ids determine.  Ids that a list or an entry's position has no room for are summed after those before them, onto
// what the matrix then holds.  Rows are dealt to workgroups by v mod R because ids are usually ranked by frequency:
// neighbours are alike in weight.
//
// Bound by memory: N d elements read, the matrix written (or the rows of tokens that occur read and written).  8192 ids, 32768 x 512 in
// fp32: 21 us (84 MB, 4.0 TB/s); 4800 ids, 32768 x 410 in bf16: 23 us (58 MB).  Where one token makes up much of the ids, by the workgroups
// that own its row, at about 12 bytes/ns each (the lines a CU has under way): 8192 ids, a quarter of them one token, added to 50257 x
// 1024: 24 to 28 us with the ids (50 MB), 9 of which go to finding and sorting the entries.  Without a workspace no others can share them.
#include "common.h"
#include "embed_sample.h"
#include "unaligned.h"

#include <algorithm>

namespace ouro {

constexpr int ES_THREADS = 512, ES_WAVES = ES_THREADS / 64;
constexpr int ES_TEAMS = ES_THREADS / STRIP_LANES;         // a team is the lanes of a strip: 128 bytes of a row of dh
constexpr int ES_STEP = 256;                               // ids of a wave at a time, four neighbours a lane
constexpr int ES_WAVE_CAP = 3 * ES_STEP, ES_CAP = ES_WAVES * ES_WAVE_CAP;     // entries of the list, of which each wave fills its part
constexpr int ES_RANK = ES_THREADS;                        // longest list that is sorted from runs of 64
constexpr int ES_COUNT = 128;                              // longest list that is sorted by counting alone (its cost grows with the square: 128 entries 1.5 us, 400 5.5
                                                           // against 3.5 from runs)
constexpr int ES_BITS = 9, ES_BINS = 1 << ES_BITS;         // largest digit of the radix sort
constexpr int ES_ROW_BITS = 14;                            // matrix rows of a workgroup: a bit each, two digits
constexpr int ES_HOT = 4096;                               // ids of one token from which on they are summed without a list, looked for among more than
                                                           // four times as many (looking takes 2 us; 60 % of 32768 ids, 1024 columns, fp32: 148 -> 77 us,
                                                           // bf16: 245 -> 157; of 16384: as before)
constexpr int ES_COLD_COST = 3;                            // rows summed in the time of one that is a sum by itself
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

// How many lanes below this one are in the set.
__device__ __forceinline__ int es_below(uint64_t set) {
  return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(set >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)set, 0));
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

// A token of the workgroup's rows that makes up ES_HOT ids and more by a sample of 64 of them, or -1 (every wave finds the same).
__device__ __forceinline__ int es_hot(const EmbedSortedParams& p, uint32_t R, uint32_t mine) {
  const int lane = threadIdx.x & 63, id = p.tok[es_sample_at(lane, p.N)];
  const bool on = (uint32_t)id < (uint32_t)p.vocab && ((uint32_t)id & (R - 1)) == mine;
  uint32_t best = (uint32_t)__popcll(es_peers((uint32_t)id, 31, __ballot(on))) << 6 | (uint32_t)lane;
  if (!on) best = 0;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) best = max(best, (uint32_t)__shfl_xor((int)best, o, 64));
  const int hot = __shfl(id, (int)(best & 63), 64);
  return (long)(best >> 6) * p.N >= 64l * ES_HOT ? __builtin_amdgcn_readfirstlane(hot) : -1;
}
// This lane's columns of the sum of the rows of token `hot`: each wave goes through its ids and sums the rows as it finds them, eight at a
// time a team.  `list`: the wave's, ES_WAVE_CAP entries; the sums of the teams are left in `heads`.
template <typename T, bool WHOLE>
__device__ __forceinline__ void es_sum_hot(const EmbedSortedParams& p, const LaneColumns& own, int hot, int wave, uint32_t* list, float* heads) {
  constexpr int P = 16 / sizeof(T), U = 8, ROUND = U * 64 / STRIP_LANES;
  static_assert(ES_WAVE_CAP >= 2 * ES_STEP + ROUND, "what is left of a round and two steps");
  const int lane = threadIdx.x & 63, team = lane / STRIP_LANES;
  const T* dh = reinterpret_cast<const T*>(p.dh) + own.col;
  float acc[P] = {};
  int4 v[2];
#pragma unroll
  for (int u = 0; u < 2; ++u) v[u] = es_ids(p, (wave * 2 + u) * ES_STEP + 4 * lane);
  int k = 0;
  for (int n = wave * 2 * ES_STEP; n < p.N; n += ES_WAVES * 2 * ES_STEP) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      auto take = [&](int id, int at) __attribute__((always_inline)) {
        const uint64_t all = __ballot(id == hot);
        if (id == hot) list[k + es_below(all)] = (uint32_t)at;
        k += (int)__popcll(all);
      };
      const int at = n + u * ES_STEP + 4 * lane;
      take(v[u].x, at); take(v[u].y, at + 1); take(v[u].z, at + 2); take(v[u].w, at + 3);
      v[u] = es_ids(p, at + ES_WAVES * 2 * ES_STEP);
    }
    __builtin_amdgcn_wave_barrier();
    const bool last = n + ES_WAVES * 2 * ES_STEP >= p.N;
    int r = 0;
    for (; r + ROUND <= k; r += ROUND) {
      UnalignedPack<T, P> x[U] = {};
#pragma unroll
      for (int u = 0; u < U; ++u) load_raw_columns<T, P, WHOLE>(dh + (size_t)list[r + u * (64 / STRIP_LANES) + team] * p.lddh, x[u], own.n);
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int j = 0; j < P; ++j) acc[j] += to_f32(x[u].v[j]);
    }
    if (last) {
      for (int i = r + team; i < k; i += 64 / STRIP_LANES) {
        UnalignedPack<T, P> x = {};
        load_raw_columns<T, P, WHOLE>(dh + (size_t)list[i] * p.lddh, x, own.n);
#pragma unroll
        for (int j = 0; j < P; ++j) acc[j] += to_f32(x.v[j]);
      }
    } else if (r > 0) {                                    // what is left, to the front
      k -= r;
      const uint32_t e = lane < k ? list[r + lane] : 0;
      __builtin_amdgcn_wave_barrier();
      if (lane < k) list[lane] = e;
      __builtin_amdgcn_wave_barrier();
    }
  }
#pragma unroll
  for (int j = 0; j < P; ++j) heads[(wave * (64 / STRIP_LANES) + team) * STRIP_LANES * P + lane % STRIP_LANES * P + j] = acc[j];
}

// WHOLE: see lane_columns.  ADD: onto what the matrix holds.
template <typename T, bool WHOLE, bool ADD>
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
  const uint32_t block = blockIdx.x - p.clearers, R = 1u << p.log2R, mine = block / p.slices;
  const LaneColumns own = lane_columns<P, WHOLE>(block % p.slices, lane % STRIP_LANES, p.d);
  const int team = tid / STRIP_LANES;
  for (int i = tid; i < 1 << max(0, p.row_bits - 5); i += ES_THREADS) seen[i] = 0;

  // ---- a token of very many ids, which no list holds: its rows are summed in the order of the ids in a team, as they are found
  const int hot = p.N > 4 * ES_HOT ? es_hot(p, R, mine) : -1;
  if (hot >= 0) {
    float* heads = reinterpret_cast<float*>(hist_or_heads);
    es_sum_hot<T, WHOLE>(p, own, hot, wave, list_a + wave * ES_WAVE_CAP, heads);
    __syncthreads();
    if (team == 0) {
      float acc[P] = {}, old[P] = {};
      float* out = p.dV + (size_t)hot * p.ldv + own.col;
      if (ADD) load_columns<float, P, WHOLE>(out, old, own.n);
      for (int t = 0; t < ES_TEAMS; ++t)
#pragma unroll
        for (int j = 0; j < P; ++j) acc[j] += heads[t * W + lane * P + j];
#pragma unroll
      for (int j = 0; j < P; ++j) old[j] = fmaf(p.scale, acc[j], old[j]);
      store_columns<float, P, WHOLE>(out, old, own.n);
    }
  }

  bool first = true, end = false;
  int n0 = 0;                                              // ids before n0 have been looked at
  while (!end) {
    // ---- the entries among the ids, in order for each wave
    const int n_base = n0;
    int k = 0;
    for (bool full = false; !full;) {
      constexpr int AHEAD = 4;                             // steps requested together
      int4 v[AHEAD];
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) v[u] = es_ids(p, n0 + (u * ES_WAVES + wave) * ES_STEP + 4 * lane);
#pragma unroll
      for (int u = 0; u < AHEAD; ++u) {
        end = n0 >= p.N;
        const int gone = n0 - n_base;
        // (a step before the positions end: no entry has all bits set, which stands for none where runs are sorted)
        full = full || end || gone >= (1 << p.n_bits) - ES_WAVES * ES_STEP;
        if (!full && gone >= ES_WAVES * ES_WAVE_CAP) full = __syncthreads_or(k > ES_WAVE_CAP - ES_STEP);
        if (full) continue;
        const int at = gone + wave * ES_STEP + 4 * lane;
        auto take = [&](uint32_t id, int n) __attribute__((always_inline)) {
          const bool on = id < (uint32_t)p.vocab && (id & (R - 1)) == mine && (int)id != hot;
          const uint64_t all = __ballot(on);
          if (on) list_a[wave * ES_WAVE_CAP + k + es_below(all)] = id >> p.log2R << p.n_bits | (uint32_t)n;
          k += (int)__popcll(all);
        };
        take(v[u].x, at); take(v[u].y, at + 1); take(v[u].z, at + 2); take(v[u].w, at + 3);
        n0 += ES_WAVES * ES_STEP;
      }
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
    // ---- a stable sort by row.  One token often makes up most of a long list (padding, the most frequent token): its entries go
    // behind the others in one pass, and what is left is short.
    uint32_t *key = list_b, *other = list_a;
    int cold = m;                                          // entries that precede those of such a token
    const int part = (m + ES_THREADS - 1) / ES_THREADS * 64, e0 = min(m, wave * part), e1 = min(m, e0 + part);     // a wave's
    if (m > ES_RANK) {
      const uint32_t sample = key[(long)lane * m / 64] >> p.n_bits;
      const uint32_t votes = (uint32_t)__popcll(es_peers(sample, p.row_bits, ~0ull)) << 6 | (uint32_t)lane;
      uint32_t best = votes;
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) best = max(best, (uint32_t)__shfl_xor((int)best, o, 64));
      const uint32_t hot = (uint32_t)__shfl((int)sample, (int)(best & 63), 64);
      int mine_cold = 0;
      for (int i = e0; i < e1; i += 64) mine_cold += (int)__popcll(__ballot(i + lane < e1 && key[i + lane] >> p.n_bits != hot));
      if (lane == 0) bins[wave] = (uint32_t)mine_cold;
      __syncthreads();
      int to_cold = 0, all_cold = 0;
#pragma unroll
      for (int w = 0; w < ES_WAVES; ++w) {
        to_cold += w < wave ? (int)bins[w] : 0;
        all_cold += (int)bins[w];
      }
      if (all_cold <= ES_RANK) {
        cold = all_cold;
        int to_hot = cold + e0 - to_cold;
        for (int i = e0; i < e1; i += 64) {
          const bool on = i + lane < e1;
          const uint32_t e = on ? key[i + lane] : 0;
          const bool is_cold = e >> p.n_bits != hot;
          const uint64_t cs = __ballot(on && is_cold), hs = __ballot(on && !is_cold);
          if (on) other[is_cold ? to_cold + es_below(cs) : to_hot + es_below(hs)] = e;
          to_cold += (int)__popcll(cs);
          to_hot += (int)__popcll(hs);
        }
        uint32_t* t = key; key = other; other = t;
      }
      __syncthreads();
    }
    if (cold > 1 && cold <= ES_RANK) {
      if (cold <= ES_COUNT) {                              // the place of an entry is the number of smaller ones: no two are equal
        if (tid < cold) {
          const uint32_t e = key[tid];
          uint32_t rank = 0;
          for (int j = 0; j < cold; j += 4) {
            const uint4 o = *reinterpret_cast<const uint4*>(key + j);
            rank += (uint32_t)(o.x < e) + (uint32_t)(j + 1 < cold && o.y < e) + (uint32_t)(j + 2 < cold && o.z < e) + (uint32_t)(j + 3 < cold && o.w < e);
          }
          other[rank] = e;
        }
      } else {
        // Each wave sorts 64 entries in registers, and the place of one is the number of smaller ones in all sorted runs.
        uint32_t e = tid < cold ? key[tid] : ~0u;
        for (int k2 = 2; k2 <= 64; k2 *= 2)
          for (int o = k2 / 2; o > 0; o /= 2) {
            const uint32_t y = (uint32_t)__shfl_xor((int)e, o, 64);
            const bool up = (lane & k2) == 0, low = (lane & o) == 0;
            e = up == low ? min(e, y) : max(e, y);
          }
        hist_or_heads[tid] = e;
        __syncthreads();
        if (tid - lane < cold && e != ~0u) {
          uint32_t rank = 0;
          for (int w = 0; w < (cold + 63) / 64; w += 4) {    // runs behind the last hold ~0
            const uint32_t* run = hist_or_heads + w * 64;
            uint32_t at[4] = {};
#pragma unroll
            for (int o = 32; o > 0; o /= 2)
#pragma unroll
              for (int r = 0; r < 4; ++r) at[r] += run[r * 64 + at[r] + o - 1] < e ? o : 0;
#pragma unroll
            for (int r = 0; r < 4; ++r) rank += at[r] + (uint32_t)(run[r * 64 + at[r]] < e);
          }
          other[rank] = e;
        }
      }
      for (int i = cold + tid; i < m; i += ES_THREADS) other[i] = key[i];
      key = other;
      __syncthreads();
    } else if (cold > ES_RANK) {
      uint32_t* hist = hist_or_heads + wave * ES_BINS;     // [wave][bin]
      uint32_t *from = key, *to = other;
      const int passes = (max(1, p.row_bits) + ES_BITS - 1) / ES_BITS, digit = (max(1, p.row_bits) + passes - 1) / passes;
      for (int shift = p.n_bits; shift < p.n_bits + max(1, p.row_bits); shift += digit) {
        const uint32_t mask = (1u << digit) - 1;
        for (int i = lane; i < ES_BINS / 4; i += 64) reinterpret_cast<uint4*>(hist)[i] = make_uint4(0, 0, 0, 0);
        for (int i = e0; i < e1; i += 64) {                // how many a bin
          const bool on = i + lane < e1;
          const uint32_t bin = on ? (from[i + lane] >> shift) & mask : 0;
          const uint64_t peers = es_peers(bin, digit, __ballot(on));
          if (on && es_below(peers) == 0) hist[bin] += (uint32_t)__popcll(peers);
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
            to[place + es_below(peers)] = e;
          }
          __builtin_amdgcn_wave_barrier();
          if (on && es_below(peers) == 0) hist[bin] = place + (uint32_t)__popcll(peers);
          __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        uint32_t* t = from; from = to; to = t;
      }
      key = from;
    }
    // ---- sums: a team takes an equal piece of the sorted list
    float* heads = reinterpret_cast<float*>(hist_or_heads);    // [team][W]: a team's part of a sum that an earlier team owns
    // (with whole waves for the entries that are likely to be sums by themselves, each with a matrix row to read or write, and for the
    // rest: teams of one wave that do different things wait for each other)
    const int dear = cold < m ? cold : 0;
    const int dear_teams = dear ? 64 / STRIP_LANES * max(1, min(ES_WAVES - 1, (ES_WAVES * ES_COLD_COST * dear + m / 2) / (m + (ES_COLD_COST - 1) * dear))) : 0;
    const bool is_dear = team < dear_teams;
    const int p0 = is_dear ? 0 : dear, p1 = is_dear ? dear : m, nth = is_dear ? team : team - dear_teams, of = is_dear ? dear_teams : ES_TEAMS - dear_teams;
    const int per = (p1 - p0 + of - 1) / of, s = min(p1, p0 + nth * per), e = min(p1, s + per);
    const uint32_t mask_n = (1u << p.n_bits) - 1;
    float acc[P] = {}, old[P] = {};                        // of the sum under way; what the matrix holds
    auto place = [&](uint32_t r) __attribute__((always_inline)) { return p.dV + ((size_t)r << p.log2R | mine) * p.ldv + own.col; };
    auto write = [&](uint32_t r) __attribute__((always_inline)) {
      if (!ADD && !first && (seen[r >> 5] >> (r & 31) & 1)) load_columns<float, P, WHOLE>(place(r), old, own.n);
#pragma unroll
      for (int j = 0; j < P; ++j) old[j] = fmaf(p.scale, acc[j], old[j]);
      store_columns<float, P, WHOLE>(place(r), old, own.n);
    };
    bool pending = false, middle = false;                  // the last sum goes on in the next team's piece, and began here or before
    uint32_t cur = 0;
    if (s < e) {
      const T* dh = reinterpret_cast<const T*>(p.dh) + n_base * p.lddh + own.col;
      cur = key[s] >> p.n_bits;
      bool head = s > p0 && key[s - 1] >> p.n_bits == cur;
      uint32_t before = head ? cur : ~0u;                  // row of the entry before the ones requested
      constexpr int U = ADD && P == 8 ? 4 : 8;             // rows requested together (within 128 registers), with the matrix rows of sums that begin
      for (int i = s; i < e; i += U) {
        UnalignedPack<T, P> x[U] = {};
        if (i > s && i + U <= e && key[i + U - 1] >> p.n_bits == cur) {      // the sum under way goes on: nothing but loads and additions
#pragma unroll
          for (int u = 0; u < U; ++u) load_raw_columns<T, P, WHOLE>(dh + (size_t)(key[i + u] & mask_n) * p.lddh, x[u], own.n);
#pragma unroll
          for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < P; ++j) acc[j] += to_f32(x[u].v[j]);
          before = cur;
          continue;
        }
        UnalignedPack<float, P> had[ADD ? U : 1] = {};
        uint32_t r[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const uint32_t entry = key[min(i + u, e - 1)];
          r[u] = entry >> p.n_bits;
          if (i + u < e) {
            load_raw_columns<T, P, WHOLE>(dh + (size_t)(entry & mask_n) * p.lddh, x[u], own.n);
            if (ADD && r[u] != before) load_raw_columns<float, P, WHOLE>(place(r[u]), had[ADD ? u : 0], own.n);
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
              for (int j = 0; j < P; ++j) { acc[j] = 0.f; old[j] = ADD ? had[ADD ? u : 0].v[j] : 0.f; }
            }
#pragma unroll
            for (int j = 0; j < P; ++j) acc[j] += to_f32(x[u].v[j]);
          }
      }
      const bool goes_on = e < p1 && key[e] >> p.n_bits == cur;
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
  p.clearers = accumulate ? 0 : (int)std::min((vocab + 3ll) / 4, std::max((long long)ES_CLEARERS, (vocab + 32ll * ES_CAP - 1) / (32ll * ES_CAP)));
  p.zero_rows = accumulate ? 0 : (int)((vocab - 1ll + p.clearers) / p.clearers);
  while (((long long)p.slices << (p.log2R + 1)) <= (accumulate ? 512 : 256) && (4ll << p.log2R) < vocab) ++p.log2R;
  while ((1ll << ES_ROW_BITS << p.log2R) < vocab) ++p.log2R;
  while ((1ll << p.row_bits << p.log2R) < vocab) ++p.row_bits;
  p.n_bits = std::min(30, 32 - p.row_bits);
  const long long blocks = ((long long)p.slices << p.log2R) + p.clearers;
  if (blocks * ES_THREADS >> 32) return hipErrorInvalidValue;
  dim3 grid((unsigned)blocks), block(ES_THREADS);
#define OURO_LAUNCH(T_, WHOLE_)                                                                                              \
  do {                                                                                                                       \
    if (accumulate) hipLaunchKernelGGL((embed_bwd_sorted_kernel<T_, WHOLE_, true>), grid, block, 0, s, p);                   \
    else hipLaunchKernelGGL((embed_bwd_sorted_kernel<T_, WHOLE_, false>), grid, block, 0, s, p);                             \
  } while (0)
  if (dtype == 1 && d >= 8) OURO_LAUNCH(bf16_t, true);
  else if (dtype == 1) OURO_LAUNCH(bf16_t, false);
  else if (d >= 4) OURO_LAUNCH(float, true);
  else OURO_LAUNCH(float, false);
#undef OURO_LAUNCH
  return hipGetLastError();
}

}  // namespace ouro
