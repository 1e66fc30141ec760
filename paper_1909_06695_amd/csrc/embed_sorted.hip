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

namespace ouro {

constexpr int ES_THREADS = 512, ES_WAVES = ES_THREADS / 64;
constexpr int ES_LANES = 8;                                // lanes of a team: 128 bytes of a row of dh
constexpr int ES_TEAMS = ES_THREADS / ES_LANES;
constexpr int ES_CAP = 2048;                               // entries of the list; more ids than that go in parts
constexpr int ES_RANK = ES_THREADS;                        // longest list that is sorted by counting smaller entries
constexpr int ES_BITS = 9, ES_BINS = 1 << ES_BITS;         // digit of the radix sort
constexpr int ES_ROWS_MAX = 1 << 14;                       // matrix rows of a workgroup (one bit each, two digits)
static_assert(ES_CAP % ES_THREADS == 0 && ES_BINS == ES_THREADS, "one bin a thread");

struct EmbedSortedParams {
  const int32_t* tok; const void* dh; float* dV;
  size_t lddh, ldv;
  int N, d, vocab;
  int log2R;
  float scale;
  int accumulate;
};

// Lanes of the wave whose `key` (bits wide) equals this lane's, among those of `in`.
__device__ __forceinline__ uint64_t es_peers(uint32_t key, int bits, uint64_t in) {
  for (int b = 0; b < bits; ++b) {
    const uint64_t set = __ballot((key >> b) & 1);
    in &= (key >> b) & 1 ? set : ~set;
  }
  return in;
}

// WHOLE: d is a whole number of 16-byte pieces of dh.
template <typename T, bool WHOLE>
__global__ __launch_bounds__(ES_THREADS) void embed_bwd_sorted_kernel(EmbedSortedParams p) {
  constexpr int P = 16 / sizeof(T);                        // columns of a lane
  constexpr int W = ES_LANES * P;                          // columns of the workgroup
  __shared__ uint32_t row_a[ES_CAP], n_a[ES_CAP], row_b[ES_CAP], n_b[ES_CAP];
  __shared__ uint32_t touched[ES_ROWS_MAX / 32];
  __shared__ __align__(16) uint32_t hist_or_heads[ES_WAVES * ES_BINS];
  __shared__ uint32_t wave_n[ES_WAVES];
  static_assert(ES_TEAMS * W <= ES_WAVES * ES_BINS, "the heads fit the histogram's place");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t R = 1u << p.log2R, mine = blockIdx.x & (R - 1);
  const int col = (blockIdx.x >> p.log2R) * W + (tid & (ES_LANES - 1)) * P;
  const int ncol = max(0, min(P, p.d - col));
  const int rows = (int)(((uint32_t)p.vocab - mine + R - 1) >> p.log2R);      // mine < vocab
  const int team = tid / ES_LANES;
  const uint64_t below = (1ull << lane) - 1;
  const bool overwrite = !p.accumulate;
  if (overwrite)
    for (int i = tid; i < (rows + 31) / 32; i += ES_THREADS) touched[i] = 0;

  // The ids [n0, n1) a wave looks at, 256 at a time: four neighbours a lane.
  auto ids = [&](int n0, int n1, auto&& take) __attribute__((always_inline)) {
    for (int n = n0; n < n1; n += 256) {
      const int at = n + 4 * lane;
      int v[4] = {-1, -1, -1, -1};
      if (at + 4 <= n1) load_unaligned<int32_t, 4>(p.tok + at, v);
      else
        for (int j = 0; j < 4; ++j)
          if (at + j < n1) v[j] = p.tok[at + j];
#pragma unroll
      for (int j = 0; j < 4; ++j) take(at + j, (uint32_t)v[j], (uint32_t)v[j] < (uint32_t)p.vocab && ((uint32_t)v[j] & (R - 1)) == mine);
    }
  };
  // Puts the entries among the ids [c0, c1) into row_a, n_a and returns their number (in every thread); with count_only only counts.
  auto collect = [&](int c0, int c1, bool count_only) __attribute__((always_inline)) {
    const int per = ((c1 - c0 + ES_WAVES - 1) / ES_WAVES + 3) & ~3;
    const int n0 = min(c1, c0 + wave * per), n1 = min(c1, n0 + per);
    uint32_t k = 0;
    ids(n0, n1, [&](int, uint32_t, bool on) { k += (uint32_t)__popcll(__ballot(on)); });
    if (lane == 0) wave_n[wave] = k;
    __syncthreads();
    uint32_t at = 0, total = 0;
    for (int w = 0; w < ES_WAVES; ++w) {
      if (w == wave) at = total;
      total += wave_n[w];
    }
    if (!count_only && total <= ES_CAP)
      ids(n0, n1, [&](int n, uint32_t v, bool on) {
        const uint64_t m = __ballot(on);
        if (on) {
          const uint32_t slot = at + (uint32_t)__popcll(m & below);
          row_a[slot] = v >> p.log2R;
          n_a[slot] = (uint32_t)n;
        }
        at += (uint32_t)__popcll(m);
      });
    __syncthreads();
    return (int)total;
  };

  bool first = true;
  int chunk = p.N;
  for (int c0 = 0; c0 < p.N || first; c0 += chunk) {
    int m = collect(c0, min(p.N, c0 + chunk), false);
    if (m > ES_CAP) {                                      // more than the list holds: in parts that cannot be
      chunk = ES_CAP;
      m = collect(c0, min(p.N, c0 + chunk), false);
    }
    // ---- stable sort by row
    const uint32_t *row = row_a, *ns = n_a;
    if (m > 1 && m <= ES_RANK) {
      if (tid < m) {
        const uint32_t r = row_a[tid];
        uint32_t rank = 0;
        for (int j = 0; j < m; ++j) rank += (uint32_t)(row_a[j] < r || (row_a[j] == r && j < tid));
        row_b[rank] = r;
        n_b[rank] = n_a[tid];
      }
      row = row_b; ns = n_b;
      __syncthreads();
    } else if (m > ES_RANK) {
      uint32_t* hist = hist_or_heads;                      // [wave][bin]
      const int per = (m + ES_THREADS - 1) / ES_THREADS * 64, e0 = min(m, wave * per), e1 = min(m, e0 + per);
      uint32_t *ra = row_a, *na = n_a, *rb = row_b, *nb = n_b;
      for (int shift = 0; shift == 0 || ((rows - 1) >> shift) > 0; shift += ES_BITS) {
        for (int i = tid; i < ES_WAVES * ES_BINS; i += ES_THREADS) hist[i] = 0;
        __syncthreads();
        for (int i = e0 + lane; i < e1; i += 64) atomicAdd(&hist[wave * ES_BINS + ((ra[i] >> shift) & (ES_BINS - 1))], 1u);
        __syncthreads();
        uint32_t sum = 0;                                  // this thread's bin over the waves, then over the bins before
        for (int w = 0; w < ES_WAVES; ++w) sum += hist[w * ES_BINS + tid];
        uint32_t incl = sum;
        for (int o = 1; o < 64; o <<= 1) {
          const uint32_t y = __shfl_up(incl, o, 64);
          if (lane >= o) incl += y;
        }
        if (lane == 63) wave_n[wave] = incl;
        __syncthreads();
        uint32_t base = incl - sum;
        for (int w = 0; w < wave; ++w) base += wave_n[w];
        for (int w = 0; w < ES_WAVES; ++w) {
          const uint32_t k = hist[w * ES_BINS + tid];
          hist[w * ES_BINS + tid] = base;
          base += k;
        }
        __syncthreads();
        for (int i0 = e0; i0 < e1; i0 += 64) {
          const bool on = i0 + lane < e1;
          const uint32_t r = on ? ra[i0 + lane] : 0, n = on ? na[i0 + lane] : 0, bin = (r >> shift) & (ES_BINS - 1);
          const uint64_t peers = es_peers(bin, ES_BITS, __ballot(on));
          if (on) {
            const uint32_t at = hist[wave * ES_BINS + bin] + (uint32_t)__popcll(peers & below);
            rb[at] = r;
            nb[at] = n;
          }
          __builtin_amdgcn_wave_barrier();
          if (on && !(peers & below)) hist[wave * ES_BINS + bin] += (uint32_t)__popcll(peers);
          __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
        uint32_t* t = ra; ra = rb; rb = t;
        t = na; na = nb; nb = t;
      }
      row = ra; ns = na;
    }
    // ---- rows without a token
    if (first && overwrite) {
      for (int i = tid; i < m; i += ES_THREADS) atomicOr(&touched[row[i] >> 5], 1u << (row[i] & 31));
      __syncthreads();
      const float zero[P] = {};
      for (int i = team; i < rows; i += ES_TEAMS)
        if (!(touched[i >> 5] >> (i & 31) & 1)) store_columns<float, P, WHOLE>(p.dV + ((size_t)i << p.log2R | mine) * p.ldv + col, zero, ncol);
    }
    // ---- sums
    float* heads = reinterpret_cast<float*>(hist_or_heads);    // [team][W]: a team's part of a sum that an earlier team owns
    const int per = (m + ES_TEAMS - 1) / ES_TEAMS, s = min(m, team * per), e = min(m, s + per);
    float acc[P] = {};
    auto write = [&](uint32_t r) __attribute__((always_inline)) {
      float* out = p.dV + ((size_t)r << p.log2R | mine) * p.ldv + col;
      float v[P] = {};
      if (!overwrite || !first) load_columns<float, P, WHOLE>(out, v, ncol);
#pragma unroll
      for (int j = 0; j < P; ++j) v[j] = fmaf(p.scale, acc[j], v[j]);
      store_columns<float, P, WHOLE>(out, v, ncol);
    };
    bool pending = false;                                  // the last sum goes on in the next team's piece
    if (s < e) {
      const T* dh = reinterpret_cast<const T*>(p.dh) + col;
      uint32_t cur = row[s];
      bool head = s > 0 && row[s - 1] == cur;
      auto flush = [&]() __attribute__((always_inline)) {
        if (head) {
#pragma unroll
          for (int j = 0; j < P; ++j) heads[team * W + (tid & (ES_LANES - 1)) * P + j] = acc[j];
        } else {
          write(cur);
        }
        head = false;
#pragma unroll
        for (int j = 0; j < P; ++j) acc[j] = 0.f;
      };
      constexpr int U = 8;                                 // rows requested together
      for (int i = s; i < e; i += U) {
        float x[U][P] = {};
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i + u < e) load_columns<T, P, WHOLE>(dh + ns[i + u] * p.lddh, x[u], ncol);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (i + u < e) {
            const uint32_t r = row[i + u];
            if (r != cur) { flush(); cur = r; }
#pragma unroll
            for (int j = 0; j < P; ++j) acc[j] += x[u][j];
          }
      }
      pending = e < m && row[e] == cur && !head;
      if (!pending) flush();
    }
    __syncthreads();
    if (pending) {
      const uint32_t cur = row[e];
      for (int t = team + 1;; ++t) {
#pragma unroll
        for (int j = 0; j < P; ++j) acc[j] += heads[t * W + (tid & (ES_LANES - 1)) * P + j];
        const int end = (t + 1) * per;
        if (end >= m || row[end] != cur) break;
      }
      write(cur);
    }
    first = false;
    __syncthreads();
    if (chunk >= p.N) break;
  }
}

hipError_t launch_embed_bwd_sorted(hipStream_t s, int dtype, const int32_t* tok, const void* dh, int lddh, float* dV, int ldv, int N, int d,
                                   int vocab, float scale, int accumulate) {
  EmbedSortedParams p;
  memset(&p, 0, sizeof p);
  p.tok = tok; p.dh = dh; p.dV = dV; p.lddh = lddh; p.ldv = ldv; p.N = N; p.d = d; p.vocab = vocab; p.scale = scale; p.accumulate = accumulate;
  const int W = ES_LANES * 16 / (dtype == 1 ? 2 : 4), slices = (d + W - 1) / W;
  // About 1024 workgroups, four matrix rows each at least; as many as keep a workgroup's rows within its bit map.
  while (((long long)slices << p.log2R) < 1024 && (4ll << p.log2R) < vocab) ++p.log2R;
  while (((long long)ES_ROWS_MAX << p.log2R) < vocab) ++p.log2R;
  const long long blocks = (long long)slices << p.log2R;
  if (blocks * ES_THREADS >> 32) return hipErrorInvalidValue;
  dim3 grid((unsigned)blocks), block(ES_THREADS);
  if (dtype == 1) {
    if (d % 8 == 0) hipLaunchKernelGGL((embed_bwd_sorted_kernel<bf16_t, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((embed_bwd_sorted_kernel<bf16_t, false>), grid, block, 0, s, p);
  } else {
    if (d % 4 == 0) hipLaunchKernelGGL((embed_bwd_sorted_kernel<float, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((embed_bwd_sorted_kernel<float, false>), grid, block, 0, s, p);
  }
  return hipGetLastError();
}

}  // namespace ouro
