// Orthogonalised updates: X = U / (|U|_F + eps), then steps of X <- a X + (b A + c A^2) X with A = X X^T, which drive the singular
// values of U towards 1 and leave its singular vectors (Newton-Schulz with the quintic whose coefficients are below, which Jordan et al.
// published for orthogonalised momentum in 2024).  U is the gradient or its momentum.
//
// The products run on fp16 matrix instructions with every operand as a sum of two fp16 numbers, high + low (22 bits of
// mantissa): x y = xh yh + xh yl + xl yh with fp32 accumulation.  One fp16 (or bf16) number is not enough: a step multiplies small singular
// values by a, five steps by 485, and with them the rounding noise of X: with 16 strong directions over noise of 1e-4 one
// fp16 number gives an error of 4.5e-2, bf16 0.37, the two halves 8e-6 and fp32 arithmetic 5e-6 (random matrices: 1.4e-3, 1.1e-2,
// 2.6e-7, 1.7e-7).  On the device, against fp32 products of the library: 0.6 to 0.9 times their error where the matrix is a few hundred wide, 1.5 times at
// 1024 x 4096 (6.3e-6 against 4.1e-6).  The fourth product, low x low, would cost a third more; it is at most 2^-22 of the whole, as much as rounding the low
// halves costs.  All entries of X, A and the polynomials are below 12 in magnitude (|X|_2 <= 1.2, |C|_2 <= 3.5); they are stored times 2^12, so that
// the low halves of ordinary entries (1 / sqrt(rows cols)) stay above fp16's smallest normal number.
//
// With C = a I + b A + c A^2 a step is X <- C X, and the A of the step after it is C A C: all of these are polynomials of one symmetric
// matrix, symmetric and commuting.  Two steps therefore need X only once: A = X X^T, C, (C A) C = A', C', C' C, X <- (C' C) X.  For
// matrices twice as wide as high and more that is a quarter to a third less work, and X is written half as often (1024 x 4096: two steps
// 2.0 -> 1.4 ms).  It is as accurate: errors of A' are absolute, 2^-22 |A|, and reach X through C' as 1e-6 of a.  Three steps without X
// would not be: negative rounding noise in the small eigenvalues of A grows by a^2 a step.
//
// Bound by the matrix instructions where matrices are large: 24 of 1024 x 4096, five steps, 3.75 ms, three times 1.21 TFLOP at 0.97 PFLOP/s.  A
// library product of 8192^3 reaches 1.54 in fp16 (1.62 in bf16, this main loop with bf16 operands 1.45).  The products with X run at 1.13 of that; the
// symmetric ones at 0.76, counting half of each: 10 whole 256 wide tiles hold the 8 that are needed, 240 of them for 256 CUs.  Bound by the latency of 17 dependent
// products where matrices are small (four of 2100 x 410: 221 us).
//
// All products are of the form L R^T with the contraction contiguous in both: X X^T; products of two of the symmetric matrices; and one of
// those times X^T, for which X is kept in both layouts.  Of the symmetric results only the tiles on and below the diagonal are formed, and
// stored twice.  Matrices are the smaller dimension times the larger, padded with zeros to whole multiples of 64: zero rows and columns
// stay zero in every step.
#include "gemm_pp.h"
#include "unaligned.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace ouro {

typedef _Float16 half_t;
typedef f16x8 half8;
typedef __attribute__((ext_vector_type(4))) _Float16 half4;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float NS_SCALE = 4096.f, NS_DOWN = 1.f / 4096.f;
constexpr int NS_NORM_PARTS = 256;                         // most partial sums of squares of a matrix
constexpr int NS_ARRIVED = 4 * 128;                        // counters: of the waves of up to 128 tiles

// A split matrix [rows][cols], cols a multiple of 32: a row holds per 32 columns the 32 high halves, then the 32 low ones.
__device__ __forceinline__ size_t ns_at(int row, int col, int cols) {
  return (size_t)row * cols * 4 + (size_t)(col >> 5) * 128 + (col & 31) * 2;
}
__device__ __forceinline__ void ns_split(float v, half_t& hi, half_t& lo) {
  hi = (half_t)v;
  lo = (half_t)(v - (float)hi);
}

struct NsParams {
  int rows, cols;                                          // of the caller's matrices
  int tall;                                                // rows > cols: X is the transpose
  int m, n, mp, np;                                        // X [m][n], m <= n; padded
  const void* g; size_t ldg; long long sg;
  float* mom; float mu; int nesterov;
  void* o; size_t ldo; long long so;
  float scale, eps;
  int parts;
  double* sums;                                            // [batch][parts]
  unsigned* arrived;                                       // [NS_ARRIVED]: see NsProduct; 0 between launches
  char *x, *xt[2], *gram, *c, *t;                          // split matrices, batch after batch
};

// ------------------------------------------------------------------------- norm, momentum
// What is orthogonalised, from the gradient and the updated momentum.
__device__ __forceinline__ float ns_update(const NsParams& p, float g, float mom) { return !p.mom ? g : p.nesterov ? fmaf(p.mu, mom, g) : mom; }

// Momentum, and the sum of squares in 64 bits: no gradient is too large or too small for it.
template <typename T>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsParams p) {
  constexpr int P = 16 / sizeof(T);
  __shared__ double part[4];
  const int b = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (blockIdx.x == 0 && b == 0)
    for (int i = threadIdx.x; i < NS_ARRIVED; i += 256) p.arrived[i] = 0;
  const T* g = reinterpret_cast<const T*>(p.g) + b * p.sg;
  float* mom = p.mom ? p.mom + b * p.sg : nullptr;
  double sum = 0;
  auto one = [&](size_t at, float x) __attribute__((always_inline)) {
    float m = 0.f;
    if (mom) mom[at] = m = fmaf(p.mu, mom[at], x);
    const double u = ns_update(p, x, m);
    sum += u * u;
  };
  for (int r = blockIdx.x * 4 + wave; r < p.rows; r += p.parts * 4) {
    const size_t row = r * p.ldg;
    const int whole = p.cols / P * P;
#pragma unroll 2
    for (int c = lane * P; c < whole; c += 64 * P) {
      T x[P];
      load_unaligned<T, P>(g + row + c, x);
      if (mom) {
#pragma unroll
        for (int h = 0; h < P; h += 4) {
          float m[4];
          load_unaligned<float, 4>(mom + row + c + h, m);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            m[e] = fmaf(p.mu, m[e], to_f32(x[h + e]));
            const double u = ns_update(p, to_f32(x[h + e]), m[e]);
            sum += u * u;
          }
          store_unaligned<float, 4>(mom + row + c + h, m);
        }
      } else {
#pragma unroll
        for (int e = 0; e < P; ++e) {
          const double u = to_f32(x[e]);
          sum += u * u;
        }
      }
    }
    if (whole + lane < p.cols) one(row + whole + lane, to_f32(g[row + whole + lane]));
  }
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (lane == 0) part[wave] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.sums[(size_t)b * p.parts + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// What U is multiplied by, in 64 bits as the sum of squares.
__device__ __forceinline__ double ns_factor(const NsParams& p, double squares) { return NS_SCALE / (sqrt(squares) + p.eps); }

// X and its transpose, split and padded, from 64 x 64 tiles.
template <typename T>
__global__ __launch_bounds__(256) void ns_start_kernel(NsParams p) {
  constexpr int P = 16 / sizeof(T);
  __shared__ float tile[64][65];
  __shared__ double part[4];
  const int tid = threadIdx.x, b = blockIdx.y, tiles_n = p.np / 64;
  const int r0 = blockIdx.x / tiles_n * 64, c0 = blockIdx.x % tiles_n * 64;    // of X
  const T* g = reinterpret_cast<const T*>(p.g) + b * p.sg;
  const float* mom = p.mom ? p.mom + b * p.sg : nullptr;
  const int i0 = p.tall ? c0 : r0, j0 = p.tall ? r0 : c0;                      // of the caller's matrix
  float u[16 / P][P];
#pragma unroll
  for (int k = 0; k < 16 / P; ++k) {
    const int at = tid + 256 * k, i = i0 + at / (64 / P), j = j0 + at % (64 / P) * P;
    T x[P] = {};
    float m[P] = {};
    if (i < p.rows) {
      if (j + P <= p.cols) {
        load_unaligned<T, P>(g + i * p.ldg + j, x);
        if (mom)
#pragma unroll
          for (int h = 0; h < P; h += 4) load_unaligned<float, 4>(mom + i * p.ldg + j + h, m + h);
      } else {
#pragma unroll
        for (int e = 0; e < P; ++e)
          if (j + e < p.cols) {
            x[e] = g[i * p.ldg + j + e];
            if (mom) m[e] = mom[i * p.ldg + j + e];
          }
      }
    }
#pragma unroll
    for (int e = 0; e < P; ++e) u[k][e] = ns_update(p, to_f32(x[e]), m[e]);
  }
  double sum = tid < p.parts ? p.sums[(size_t)b * p.parts + tid] : 0;
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((tid & 63) == 0) part[tid >> 6] = sum;
  __syncthreads();
  const double inv = ns_factor(p, (part[0] + part[1]) + (part[2] + part[3]));
#pragma unroll
  for (int k = 0; k < 16 / P; ++k) {
    const int at = tid + 256 * k, i = at / (64 / P), j = at % (64 / P) * P;
#pragma unroll
    for (int e = 0; e < P; ++e) {
      const float x = (float)(u[k][e] * inv);
      if (p.tall) tile[j + e][i] = x;
      else tile[i][j + e] = x;
    }
  }
  __syncthreads();
  const size_t bytes = (size_t)p.mp * p.np * 4;
  for (int k = tid; k < 64 * 8; k += 256) {
    const int r = k >> 3, c = (k & 7) * 8;
    half8 hi, lo, thi, tlo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      half_t h, l;
      ns_split(tile[r][c + e], h, l);
      hi[e] = h; lo[e] = l;
      ns_split(tile[c + e][r], h, l);
      thi[e] = h; tlo[e] = l;
    }
    char* x = p.x + b * bytes + ns_at(r0 + r, c0 + c, p.np);
    *reinterpret_cast<half8*>(x) = hi;
    *reinterpret_cast<half8*>(x + 64) = lo;
    char* t = p.xt[0] + b * bytes + ns_at(c0 + r, r0 + c, p.mp);
    *reinterpret_cast<half8*>(t) = thi;
    *reinterpret_cast<half8*>(t + 64) = tlo;
  }
}

// ------------------------------------------------------------------------------- products
enum { NS_PLAIN = 0, NS_POLY = 1, NS_NEXT = 2, NS_LAST = 3 };     // L R^T (symmetric); a I + b L + c L L^T; X and X^T; the result
struct NsProduct {
  const char* a; const char* b;                            // split [rows_a][32 k_tiles], [rows_b][32 k_tiles], batch after batch
  int rows_a, rows_b, k_tiles;
  int tiles_b;                                             // tiles along rows_b; symmetric results: 0
  int tiles;                                               // of one matrix
  char* out; char* out_t;                                  // PLAIN, POLY: the result; NEXT: X and X^T
  // PLAIN, few tiles and a long contraction: a tile has `splits` workgroups, each a range of `per` K-tiles.  They leave their sums in `parts`, wave
  // by wave, and the wave that arrives last adds those of its piece up in order and goes on with the epilogue.
  int splits, per;
  double* parts;                                           // two sums each, [matrix][tile][split][wave][8][lane]
};

// The matrix and the tile of a workgroup.  Workgroups are dealt to the 8 XCDs in turn; an XCD takes a run of neighbouring tiles, whose
// operands its L2 then shares.
struct NsTile { int b, ti, tj, split; };       // split: of q.splits > 1
__device__ __forceinline__ NsTile ns_tile(const NsProduct& q) {
  const int nb = gridDim.x, share = nb >> 3, rest = nb & 7, xcd = blockIdx.x & 7, at = xcd * share + min(xcd, rest) + (blockIdx.x >> 3);
  const int bid = q.splits > 1 ? at / q.splits : at;
  NsTile r;
  r.split = at - bid * q.splits;
  r.b = bid / q.tiles;
  const int t = bid - r.b * q.tiles;
  if (q.tiles_b) {
    r.ti = t / q.tiles_b;
    r.tj = t - r.ti * q.tiles_b;
  } else {                                                 // row ti of the triangle begins at ti (ti + 1) / 2
    r.ti = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
    while (r.ti * (r.ti + 1) / 2 > t) --r.ti;
    while ((r.ti + 1) * (r.ti + 2) / 2 <= t) ++r.ti;
    r.tj = t - r.ti * (r.ti + 1) / 2;
  }
  return r;
}

// One 32 x 32 piece of a product at (m, n) of matrix b.  In both layouts its rows are full 128-byte lines (32 high halves, 32 low ones).
// The accumulators go through the wave's patch of LDS, [n][m] as lanes hold them, and leave first with m contiguous (where
// what is added comes from), then with n contiguous.
constexpr int NS_PATCH = 32 * 36;                          // floats
template <int KIND, typename T>
__device__ __forceinline__ void ns_epilogue(const NsParams& p, const NsProduct& q, int b, int m, int n, bool diagonal, const f32x16& acc, float* patch, int lane) {
  if (m >= q.rows_a || n >= q.rows_b) return;              // both are multiples of 64
  const size_t mat = (size_t)b * q.rows_a * q.rows_b * 4;
  const int row = lane >> 2, c = (lane & 3) * 8;
  half8 old_hi[2], old_lo[2];
  if (KIND == NS_POLY) {                                   // A itself, symmetric
#pragma unroll
    for (int it = 0; it < 2; ++it) {
      const char* old = q.a + mat + ns_at(n + 16 * it + row, m + c, q.rows_a);
      old_hi[it] = *reinterpret_cast<const half8*>(old);
      old_lo[it] = *reinterpret_cast<const half8*>(old + 64);
    }
  }
#pragma unroll
  for (int r = 0; r < 4; ++r)
    *reinterpret_cast<float4*>(patch + (lane & 31) * 36 + 8 * r + 4 * (lane >> 5)) =
        make_float4(acc[4 * r] * NS_DOWN, acc[4 * r + 1] * NS_DOWN, acc[4 * r + 2] * NS_DOWN, acc[4 * r + 3] * NS_DOWN);
  __builtin_amdgcn_wave_barrier();
  auto store_split = [](char* at, const float* v) __attribute__((always_inline)) {
    half8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      half_t h, l;
      ns_split(v[e], h, l);
      hi[e] = h; lo[e] = l;
    }
    *reinterpret_cast<half8*>(at) = hi;
    *reinterpret_cast<half8*>(at + 64) = lo;
  };
  auto store_result = [&](int i, int j, int lim_i, int lim_j, const float* v) __attribute__((always_inline)) {     // o[i][j ...]
    if (i >= lim_i) return;
    T* o = reinterpret_cast<T*>(p.o) + b * p.so + i * p.ldo + j;
    T w[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = from_f32<T>(v[e] * (p.scale * NS_DOWN));
    if (j + 8 <= lim_j) {
#pragma unroll
      for (int e = 0; e < 8; e += 16 / (int)sizeof(T)) store_unaligned<T, 16 / sizeof(T)>(o + e, w + e);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (j + e < lim_j) o[e] = w[e];
    }
  };
#pragma unroll
  for (int it = 0; it < 2; ++it) {
    float* at = patch + (16 * it + row) * 36 + c;
    float v[8];
    *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(at);
    *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(at + 4);
    if (KIND == NS_POLY) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = (float)old_hi[it][e] + (float)old_lo[it][e];
        v[e] = fmaf(NS_C, v[e], fmaf(NS_B, x, m + c + e == n + 16 * it + row ? NS_A * NS_SCALE : 0.f));
      }
      *reinterpret_cast<float4*>(at) = *reinterpret_cast<const float4*>(v);
      *reinterpret_cast<float4*>(at + 4) = *reinterpret_cast<const float4*>(v + 4);
    }
    if (KIND == NS_LAST) {
      if (p.tall) store_result(n + 16 * it + row, m + c, p.n, p.m, v);
    } else {
      store_split((KIND == NS_NEXT ? q.out_t : q.out) + mat + ns_at(n + 16 * it + row, m + c, q.rows_a), v);
    }
  }
  __builtin_amdgcn_wave_barrier();
  if (KIND == NS_LAST ? !p.tall : KIND == NS_NEXT || !diagonal) {      // a tile on the diagonal holds both of each pair
#pragma unroll
    for (int it = 0; it < 2; ++it) {
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = patch[(c + e) * 36 + 16 * it + row];
      if (KIND == NS_LAST) store_result(m + 16 * it + row, n + c, p.m, p.n, v);
      else store_split(q.out + mat + ns_at(m + 16 * it + row, n + c, q.rows_b), v);
    }
  }
  __builtin_amdgcn_wave_barrier();
}

// The fragments of a K-tile, S 32-row tiles of either operand, four chunks (high 0-15, high 16-31, low 0-15, low 16-31) each.  One block of
// assembly, with its wait: the compiler cannot tell an LDS read from the target of the direct loads in flight and would drain
// those first.
__device__ __forceinline__ void ns_read(half8 (&a)[1][4], half8 (&b)[1][4], const uint32_t* ra, const uint32_t* rb) {
  asm volatile(
      "ds_read_b128 %0, %8\n\tds_read_b128 %4, %12\n\tds_read_b128 %1, %9\n\tds_read_b128 %5, %13\n\t"
      "ds_read_b128 %2, %10\n\tds_read_b128 %6, %14\n\tds_read_b128 %3, %11\n\tds_read_b128 %7, %15\n\ts_waitcnt lgkmcnt(0)"
      : "=&v"(a[0][0]), "=&v"(a[0][1]), "=&v"(a[0][2]), "=&v"(a[0][3]), "=&v"(b[0][0]), "=&v"(b[0][1]), "=&v"(b[0][2]), "=&v"(b[0][3])
      : "v"(ra[0]), "v"(ra[1]), "v"(ra[2]), "v"(ra[3]), "v"(rb[0]), "v"(rb[1]), "v"(rb[2]), "v"(rb[3])
      : "memory");
}
__device__ __forceinline__ void ns_read(half8 (&a)[2][4], half8 (&b)[2][4], const uint32_t* ra, const uint32_t* rb) {
  asm volatile(
      "ds_read_b128 %0, %16\n\tds_read_b128 %4, %16 offset:4096\n\tds_read_b128 %8, %20\n\tds_read_b128 %12, %20 offset:4096\n\t"
      "ds_read_b128 %1, %17\n\tds_read_b128 %5, %17 offset:4096\n\tds_read_b128 %9, %21\n\tds_read_b128 %13, %21 offset:4096\n\t"
      "ds_read_b128 %2, %18\n\tds_read_b128 %6, %18 offset:4096\n\tds_read_b128 %10, %22\n\tds_read_b128 %14, %22 offset:4096\n\t"
      "ds_read_b128 %3, %19\n\tds_read_b128 %7, %19 offset:4096\n\tds_read_b128 %11, %23\n\tds_read_b128 %15, %23 offset:4096\n\t"
      "s_waitcnt lgkmcnt(0)"
      : "=&v"(a[0][0]), "=&v"(a[0][1]), "=&v"(a[0][2]), "=&v"(a[0][3]), "=&v"(a[1][0]), "=&v"(a[1][1]), "=&v"(a[1][2]), "=&v"(a[1][3]),
        "=&v"(b[0][0]), "=&v"(b[0][1]), "=&v"(b[0][2]), "=&v"(b[0][3]), "=&v"(b[1][0]), "=&v"(b[1][1]), "=&v"(b[1][2]), "=&v"(b[1][3])
      : "v"(ra[0]), "v"(ra[1]), "v"(ra[2]), "v"(ra[3]), "v"(rb[0]), "v"(rb[1]), "v"(rb[2]), "v"(rb[3])
      : "memory");
}

__device__ __forceinline__ void ns_request(const char* base, int bytes, char* dst, uint32_t voff, uint32_t k) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(base), 0, bytes, 0x00020000), (lds_void*)dst, 16, voff, k, 0, 0);
}

// 64 S x 64 S tiles, four waves of 32 S x 32 S each.  A K-tile is 32 of the contraction: 128-byte rows of high and low halves in LDS, 16-byte
// chunk c of a row at c ^ swizzle(row), in two stages filled by direct loads: a K-tile's are requested when the one before it has arrived, and are waited
// for, all of them, before the barrier that opens it.  G groups
// of four waves take every G-th K-tile each and are added up in order at the end: with one workgroup a CU a K-tile costs its latency
// (wait, barrier, fragments, six dependent matrix instructions: 0.37 us), and four at a time a quarter of it.
template <int S, int G> struct NsSmall {
  static constexpr int ROWS = 64 * S, STAGE = 2 * ROWS * 128, D = 2, LDS = G * D * STAGE;
};
template <int S, int G, int KIND, typename T>
__global__ __launch_bounds__(256 * G) void ns_product_kernel(NsParams p, NsProduct q) {
  constexpr int ROWS = NsSmall<S, G>::ROWS, STAGE = NsSmall<S, G>::STAGE, D = NsSmall<S, G>::D, PER = 4 * S;
  extern __shared__ uint4 smem[];
  static_assert(NsSmall<S, G>::LDS >= (G - 1) * 4 * S * S * 4096 + 4 * NS_PATCH * 4, "the groups' sums and the epilogue's patches fit the ring");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3, group = __builtin_amdgcn_readfirstlane(tid >> 8);
  char* const lds = reinterpret_cast<char*>(smem) + group * D * STAGE;
  const NsTile t = ns_tile(q);
  const int m0 = t.ti * ROWS, n0 = t.tj * ROWS, ld = q.k_tiles * 128;
  const int bytes_a = q.rows_a * ld, bytes_b = q.rows_b * ld;
  const char* A = q.a + (size_t)t.b * bytes_a;
  const char* B = q.b + (size_t)t.b * bytes_b;
  auto swizzle = [](int row) { return (row ^ ((row & 31) >> 3)) & 7; };
  uint32_t oa[2 * S], ob[2 * S];                           // 8 rows a request; rows past the end read as zero
#pragma unroll
  for (int i = 0; i < 2 * S; ++i) {
    const int row = (wave * 2 * S + i) * 8 + (lane >> 3);
    const uint32_t off = (uint32_t)(((lane & 7) ^ swizzle(row)) << 4);
    oa[i] = (uint32_t)(m0 + row) * ld + off;
    ob[i] = (uint32_t)(n0 + row) * ld + off;
  }
  const bool split = KIND == NS_PLAIN && S == 1 && G == 4 && q.splits > 1;
  const int k0 = split ? t.split * q.per : 0, k_tiles = split ? min(q.per, q.k_tiles - k0) : q.k_tiles;
  const int mine = (k_tiles - group + G - 1) / G, most = (k_tiles + G - 1) / G;     // K-tiles group, group + G, ...
  auto request = [&](int i, int stage) __attribute__((always_inline)) {
    char* dst = lds + stage * STAGE + wave * 2 * S * 1024;
    const uint32_t k = (uint32_t)(k0 + i * G + group) * 128;
#pragma unroll
    for (int r = 0; r < 2 * S; ++r) {
      ns_request(A, bytes_a, dst + r * 1024, oa[r], k);
      ns_request(B, bytes_b, dst + ROWS * 128 + r * 1024, ob[r], k);
    }
  };
  f32x16 acc[S][S];
#pragma unroll
  for (int i = 0; i < S * S; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[i / S][i % S][r] = 0.f;
  const int wm = (wave >> 1) * 32 * S, wn = (wave & 1) * 32 * S;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  uint32_t fa0[4], fb0[4];
#pragma unroll
  for (int c = 0; c < 4; ++c) {
    const int ra = wm + (lane & 31), rb = wn + (lane & 31), ch = 2 * c + (lane >> 5);
    fa0[c] = lds0 + ra * 128 + ((ch ^ swizzle(ra)) << 4);
    fb0[c] = lds0 + ROWS * 128 + rb * 128 + ((ch ^ swizzle(rb)) << 4);
  }
  for (int i = 0; i < D - 1 && i < mine; ++i) request(i, i);
  int stage = 0;
  for (int i = 0; i < most; ++i) {
    if (i + D - 2 < mine) pp_wait_mem<PER*(D - 2)>();      // the group's K-tile i has arrived
    else pp_wait_mem<0>();
    pp_barrier();                                          // ... for every wave, and nobody reads the stage that is filled next
    if (i + D - 1 < mine) request(i + D - 1, stage == 0 ? D - 1 : stage - 1);
    if (i < mine) {
      half8 fa[S][4], fb[S][4];
      uint32_t ra[4], rb[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) { ra[c] = fa0[c] + stage * STAGE; rb[c] = fb0[c] + stage * STAGE; }
      ns_read(fa, fb, ra, rb);
#pragma unroll
      for (int pass = 0; pass < 6; ++pass) {
        const int ca = pass >> 1 == 2 ? 2 + (pass & 1) : pass & 1, cb = pass >> 1 == 1 ? 2 + (pass & 1) : pass & 1;
#pragma unroll
        for (int r = 0; r < S * S; ++r) acc[r / S][r % S] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[r / S][ca], fb[r % S][cb], acc[r / S][r % S], 0, 0, 0);
      }
    }
    stage = stage + 1 == D ? 0 : stage + 1;
  }
  __syncthreads();
  if (G > 1) {
    float4* sums = reinterpret_cast<float4*>(smem);        // [group - 1][wave][piece][4][lane]
    if (group > 0) {
#pragma unroll
      for (int i = 0; i < S * S; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          sums[((((group - 1) * 4 + wave) * S * S + i) * 4 + r) * 64 + lane] =
              make_float4(acc[i / S][i % S][4 * r], acc[i / S][i % S][4 * r + 1], acc[i / S][i % S][4 * r + 2], acc[i / S][i % S][4 * r + 3]);
    }
    __syncthreads();
    if (group > 0) return;
    for (int g = 0; g < G - 1; ++g)
#pragma unroll
      for (int i = 0; i < S * S; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4 v = sums[(((g * 4 + wave) * S * S + i) * 4 + r) * 64 + lane];
          acc[i / S][i % S][4 * r] += v.x; acc[i / S][i % S][4 * r + 1] += v.y; acc[i / S][i % S][4 * r + 2] += v.z; acc[i / S][i % S][4 * r + 3] += v.w;
        }
  }
  if (split) {
    // (Stores and loads that pass by the caches XCDs do not share, and the counter after the stores have arrived: fences, which write back and
    // drop a whole L2, take 30 us here.)
    const size_t tile = (size_t)t.b * q.tiles + t.ti * (t.ti + 1) / 2 + t.tj;
    double* part = q.parts + ((tile * q.splits * 4 + wave) * 8) * 64 + lane;
    constexpr int APART = 4 * 8 * 64;                      // of a split
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      const float2 two = make_float2(acc[0][0][2 * r], acc[0][0][2 * r + 1]);
      __hip_atomic_store(part + t.split * APART + r * 64, __builtin_bit_cast(double, two), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    unsigned* arrived = p.arrived + tile * 4 + wave;
    unsigned nth = 0;
    if (lane == 0) nth = __hip_atomic_fetch_add(arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (__builtin_amdgcn_readfirstlane((int)nth) + 1 < q.splits) return;
    asm volatile("" ::: "memory");
    if (lane == 0) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[0][0][r] = 0.f;
#pragma unroll 4
    for (int k = 0; k < q.splits; ++k)
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const float2 two = __builtin_bit_cast(float2, __hip_atomic_load(part + k * APART + r * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
        acc[0][0][2 * r] += two.x; acc[0][0][2 * r + 1] += two.y;
      }
  }
  float* patch = reinterpret_cast<float*>(smem) + (G - 1) * 4 * S * S * 1024 + wave * NS_PATCH;      // behind the sums, which other waves may still read
#pragma unroll
  for (int i = 0; i < S * S; ++i)
    ns_epilogue<KIND, T>(p, q, t.b, m0 + wm + 32 * (i / S), n0 + wn + 32 * (i % S), t.ti == t.tj, acc[i / S][i % S], patch, lane);
}

// 256 x 256 tiles (gemm_pp.h).
template <int KIND, typename T>
__global__ __launch_bounds__(512, 2) void ns_product_pp_kernel(NsParams p, NsProduct q) {
  extern __shared__ uint4 smem[];
  static_assert(PP_LDS >= 8 * NS_PATCH * 4, "the epilogue's patches fit the ring");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const NsTile t = ns_tile(q);
  const int m0 = t.ti * 256, n0 = t.tj * 256;
  GemmParams g;                                            // what the main loop reads of it
  g.lda = g.ldb = q.k_tiles * 64;
  g.bytesA = q.rows_a * q.k_tiles * 128;
  g.bytesB = q.rows_b * q.k_tiles * 128;
  g.A = q.a + (size_t)t.b * g.bytesA;
  g.B = q.b + (size_t)t.b * g.bytesB;
  f32x16 acc[4][2];
  pp_mainloop<false, true, true>(g, m0, n0, 0, q.k_tiles, reinterpret_cast<char*>(smem), acc);
  float* patch = reinterpret_cast<float*>(smem) + wave * NS_PATCH;
  const int m_w = m0 + 64 * (wave >> 2), n_w = n0 + 32 * (wave & 3);
#pragma unroll
  for (int i = 0; i < 8; ++i)
    ns_epilogue<KIND, T>(p, q, t.b, m_w + 128 * (i >> 2) + 32 * ((i >> 1) & 1), n_w + 128 * (i & 1), t.ti == t.tj, acc[i >> 1][i & 1], patch, lane);
}

// ------------------------------------------------------------- the small products of a pair
// For m up to 64 what lies between A and C' C (or, of a single step, C) is one launch: a workgroup takes a matrix, four waves a 32 x 32 tile
// of it each, and the two matrices that are needed at a time stay in LDS.  A launch per product costs its latency, 3 to 5 us (64 x 256:
// 67 -> 49 us).  (At m = 128 the fragment reads take the LDS 2 us a product, and it gains nothing.)  Rows are as in memory, the 16-byte
// chunks of row r at c ^ (r & 15).  All tiles are formed: what is stored for (n, m) is the value of (m, n).
struct NsChain {
  static constexpr int M = 64, ROW = M * 4, BYTES = M * ROW, TILES = M / 32, THREADS = 64 * TILES * TILES;
  __device__ static __forceinline__ int at(int row, int chunk) { return row * ROW + ((chunk ^ (row & 15)) << 4); }
  // acc = the tile of L R^T
  __device__ static __forceinline__ void product(const char* l, const char* r, int ti, int tj, int lane, float (&v)[16]) {
    f32x16 big, small;                                     // high x high, and the others
#pragma unroll
    for (int i = 0; i < 16; ++i) big[i] = small[i] = 0.f;
#pragma unroll
    for (int kt = 0; kt < M / 32; ++kt) {
      half8 a[4], b[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        a[c] = *reinterpret_cast<const half8*>(l + at(32 * ti + (lane & 31), kt * 8 + 2 * c + (lane >> 5)));
        b[c] = *reinterpret_cast<const half8*>(r + at(32 * tj + (lane & 31), kt * 8 + 2 * c + (lane >> 5)));
      }
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        big = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[c], b[c], big, 0, 0, 0);
        small = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[c], b[2 + c], small, 0, 0, 0);
        small = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[2 + c], b[c], small, 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = (big[i] + small[i]) * NS_DOWN;
  }
  // v = a I + b A + c v
  __device__ static __forceinline__ void polynomial(const char* a, int ti, int tj, int lane, float (&v)[16]) {
    const int n = 32 * tj + (lane & 31);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int m = 32 * ti + 8 * r + 4 * (lane >> 5), chunk = ti * 8 + r, half = (lane >> 5) * 8;
      const half4 hi = *reinterpret_cast<const half4*>(a + at(n, chunk) + half), lo = *reinterpret_cast<const half4*>(a + at(n, chunk + 4) + half);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        v[4 * r + e] = fmaf(NS_C, v[4 * r + e], fmaf(NS_B, (float)hi[e] + (float)lo[e], m + e == n ? NS_A * NS_SCALE : 0.f));
    }
  }
  __device__ static __forceinline__ void store(char* to, int ti, int tj, int lane, const float (&v)[16]) {
    const int n = 32 * tj + (lane & 31);
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      half4 hi, lo;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        half_t h, l;
        ns_split(v[4 * r + e], h, l);
        hi[e] = h; lo[e] = l;
      }
      const int chunk = ti * 8 + r, half = (lane >> 5) * 8;
      *reinterpret_cast<half4*>(to + at(n, chunk) + half) = hi;
      *reinterpret_cast<half4*>(to + at(n, chunk + 4) + half) = lo;
    }
  }
};
// x: A, then C' C (two steps) or C, for the tile (ti, tj) of a wave that takes part; c: room for C.  All waves of the workgroup call.
__device__ __forceinline__ void ns_chain(char* x, char* c, bool two, bool part, int ti, int tj, int lane) {
  float v[16];
  auto replace = [&](char* to, const char* l, const char* r, bool poly) __attribute__((always_inline)) {      // to <- l r^T, or (l = r = x) its polynomial
    if (part) {
      NsChain::product(l, r, ti, tj, lane, v);
      if (poly) NsChain::polynomial(x, ti, tj, lane, v);
    }
    if (to == x) __syncthreads();
    if (part) NsChain::store(to, ti, tj, lane, v);
    __syncthreads();
  };
  replace(two ? c : x, x, x, true);
  if (!two) return;
#pragma unroll 1
  for (int k = 0; k < 4; ++k) replace(x, k == 0 ? c : x, k == 0 || k == 2 ? x : c, k == 2);     // C A; C A C; C'; C' C
}
__global__ __launch_bounds__(NsChain::THREADS) void ns_chain_kernel(char* gram, int two) {
  using K = NsChain;
  extern __shared__ uint4 smem[];
  char* x = reinterpret_cast<char*>(smem);
  char* g = gram + (size_t)blockIdx.x * K::BYTES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  for (int i = tid; i < K::BYTES / 16; i += K::THREADS)
    *reinterpret_cast<uint4*>(x + K::at(i / (K::ROW / 16), i % (K::ROW / 16))) = reinterpret_cast<const uint4*>(g)[i];
  __syncthreads();
  ns_chain(x, x + K::BYTES, two, true, wave / K::TILES, wave % K::TILES, lane);
  for (int i = tid; i < K::BYTES / 16; i += K::THREADS)
    reinterpret_cast<uint4*>(g)[i] = *reinterpret_cast<const uint4*>(x + K::at(i / (K::ROW / 16), i % (K::ROW / 16)));
}

// ----------------------------------------------------------------------- a matrix a workgroup
// Matrices up to 64 x 256 in one launch: a workgroup of 16 waves takes a matrix from the gradient to the result, X in LDS, a wave a 32 x 32
// tile of it.  X X^T shares its contraction among four groups of waves; C' C times X reads X with the transposing LDS read and
// replaces it in place.
constexpr int NS_ALONE_COLS = 256, NS_ALONE_WAVES = 16;
constexpr int NS_ALONE_PITCH = NS_ALONE_COLS * 4 + 16;     // bytes of a row of X: the next one 16 bytes further in the banks
constexpr int NS_ALONE_X = 64 * NS_ALONE_PITCH, NS_ALONE_SUMS = 3 * 4 * 4096;
constexpr int NS_ALONE_LDS = 2 * NsChain::BYTES + NS_ALONE_X + NS_ALONE_SUMS;
template <typename T>
__global__ __launch_bounds__(64 * NS_ALONE_WAVES) void ns_alone_kernel(NsParams p, int steps) {
  extern __shared__ uint4 smem[];
  char* const a = reinterpret_cast<char*>(smem);           // A ... C' C
  char* const c = a + NsChain::BYTES;
  char* const x = c + NsChain::BYTES;                      // [64][NS_ALONE_PITCH], rows as in memory
  float4* const sums = reinterpret_cast<float4*>(x + NS_ALONE_X);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), b = blockIdx.x;
  // ---- U / (|U| + eps): 16 values a thread
  constexpr int P = 16 / sizeof(T), CHUNKS = 16 / P;
  const T* g = reinterpret_cast<const T*>(p.g) + b * p.sg;
  float* mom = p.mom ? p.mom + b * p.sg : nullptr;
  float u[CHUNKS][P];
  double sum = 0;
  const int per_row = (p.cols + P - 1) / P;                // pieces of the caller's rows: at most 64 x 256 / P + 256 of them
#pragma unroll
  for (int k = 0; k < CHUNKS; ++k) {
    const int at = tid + 1024 * k, i = at / per_row, j = at % per_row * P;
    const int n = i < p.rows ? min(P, p.cols - j) : 0;
    const size_t o = i * p.ldg + j;
    T v[P] = {};
    if (n == P) load_unaligned<T, P>(g + o, v);
    else
#pragma unroll
      for (int e = 0; e < P - 1; ++e)
        if (e < n) v[e] = g[o + e];
#pragma unroll
    for (int e = 0; e < P; ++e) {
      float m = 0.f;
      if (mom && e < n) mom[o + e] = m = fmaf(p.mu, mom[o + e], to_f32(v[e]));
      u[k][e] = ns_update(p, to_f32(v[e]), m);
      sum += (double)u[k][e] * u[k][e];
    }
  }
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if (lane == 0) reinterpret_cast<double*>(sums)[wave] = sum;
  for (int i = tid; i < NS_ALONE_X / 16; i += 1024) reinterpret_cast<uint4*>(x)[i] = make_uint4(0, 0, 0, 0);
  __syncthreads();
  sum = 0;
  for (int w = 0; w < NS_ALONE_WAVES; ++w) sum += reinterpret_cast<double*>(sums)[w];
  const double inv = ns_factor(p, sum);
  auto put = [&](int m, int n, float v) __attribute__((always_inline)) {
    half_t hi, lo;
    ns_split(v, hi, lo);
    char* at = x + m * NS_ALONE_PITCH + (n >> 5) * 128 + (n & 31) * 2;
    *reinterpret_cast<half_t*>(at) = hi;
    *reinterpret_cast<half_t*>(at + 64) = lo;
  };
#pragma unroll
  for (int k = 0; k < CHUNKS; ++k) {
    const int at = tid + 1024 * k, i = at / per_row, j = at % per_row * P;
    if (i >= p.rows) continue;
    if (p.tall) {
#pragma unroll
      for (int e = 0; e < P; ++e)
        if (j + e < p.cols) put(j + e, i, (float)(u[k][e] * inv));
    } else {                                               // (what lies past the columns is zero)
      typedef _Float16 Piece __attribute__((ext_vector_type(P)));
      Piece hi, lo;
#pragma unroll
      for (int e = 0; e < P; ++e) {
        half_t h, l;
        ns_split((float)(u[k][e] * inv), h, l);
        hi[e] = h; lo[e] = l;
      }
      char* to = x + i * NS_ALONE_PITCH + (j >> 5) * 128 + (j & 31) * 2;
      *reinterpret_cast<Piece*>(to) = hi;
      *reinterpret_cast<Piece*>(to + 64) = lo;
    }
  }
  __syncthreads();
  const int k_tiles = p.np / 32, tile = wave & 3, group = wave >> 2;
  for (int i = 0; i < steps;) {
    const bool two = i + 1 < steps;
    // ---- A = X X^T
    f32x16 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    for (int kt = group; kt < k_tiles; kt += 4) {
      half8 l[4], r[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        l[q] = *reinterpret_cast<const half8*>(x + (32 * (tile >> 1) + (lane & 31)) * NS_ALONE_PITCH + kt * 128 + q * 32 + (lane >> 5) * 16);
        r[q] = *reinterpret_cast<const half8*>(x + (32 * (tile & 1) + (lane & 31)) * NS_ALONE_PITCH + kt * 128 + q * 32 + (lane >> 5) * 16);
      }
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[q], r[q], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[q], r[2 + q], acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(l[2 + q], r[q], acc, 0, 0, 0);
      }
    }
    if (group > 0)
#pragma unroll
      for (int r = 0; r < 4; ++r) sums[(((group - 1) * 4 + tile) * 4 + r) * 64 + lane] = make_float4(acc[4 * r], acc[4 * r + 1], acc[4 * r + 2], acc[4 * r + 3]);
    __syncthreads();
    if (group == 0) {
      float v[16];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int q = 0; q < 3; ++q) {
          const float4 o = sums[((q * 4 + tile) * 4 + r) * 64 + lane];
          acc[4 * r] += o.x; acc[4 * r + 1] += o.y; acc[4 * r + 2] += o.z; acc[4 * r + 3] += o.w;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * r + e] = acc[4 * r + e] * NS_DOWN;
      }
      NsChain::store(a, tile >> 1, tile & 1, lane, v);
    }
    __syncthreads();
    ns_chain(a, c, two, wave < 4, tile >> 1, tile & 1, lane);
    i += two ? 2 : 1;
    // ---- X <- (C' C) X: the wave's tile, 32 rows ti of the polynomial and 32 columns tj of X
    const int ti = wave & 1, tj = wave >> 1;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.f;
    if (tj < k_tiles) {
      // the transposing read: 16 lanes fetch four rows of 16 columns and get four rows of a column each
      const int g4 = lane >> 4, l16 = lane & 15;
      const uint32_t from = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)x + (8 * (g4 >> 1) + (l16 >> 2)) * NS_ALONE_PITCH + tj * 128 + 2 * (16 * (g4 & 1) + 4 * (l16 & 3));
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) {
        u32x2 r[4];
        asm volatile(
            "ds_read_b64_tr_b16 %0, %4\n\tds_read_b64_tr_b16 %1, %4 offset:%5\n\t"
            "ds_read_b64_tr_b16 %2, %4 offset:64\n\tds_read_b64_tr_b16 %3, %4 offset:%6\n\ts_waitcnt lgkmcnt(0)"
            : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3])
            : "v"(from + ks * 16 * NS_ALONE_PITCH), "n"(4 * NS_ALONE_PITCH), "n"(4 * NS_ALONE_PITCH + 64)
            : "memory");
        const half8 rh = __builtin_bit_cast(half8, __builtin_shufflevector(r[0], r[1], 0, 1, 2, 3)), rl = __builtin_bit_cast(half8, __builtin_shufflevector(r[2], r[3], 0, 1, 2, 3));
        const int chunk = (ks >> 1) * 8 + (ks & 1) * 2 + (lane >> 5);
        const half8 lh = *reinterpret_cast<const half8*>(a + NsChain::at(32 * ti + (lane & 31), chunk)), ll = *reinterpret_cast<const half8*>(a + NsChain::at(32 * ti + (lane & 31), chunk + 4));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh, rh, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(lh, rl, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ll, rh, acc, 0, 0, 0);
      }
    }
    __syncthreads();
    if (tj < k_tiles) {
      const int n = 32 * tj + (lane & 31);
      T* o = reinterpret_cast<T*>(p.o) + b * p.so;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int m = 32 * ti + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
        if (i < steps) put(m, n, acc[r] * NS_DOWN);
        else if (m < p.m && n < p.n) o[p.tall ? n * p.ldo + m : m * p.ldo + n] = from_f32<T>(acc[r] * (NS_DOWN * NS_DOWN) * p.scale);
      }
    }
    __syncthreads();
  }
}

// ---------------------------------------------------------------------------------- host
static int ns_pad(int x) { return (x + 63) / 64 * 64; }
static size_t ns_align(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t orthogonalize_scratch_floats(int batch, int rows, int cols) {
  const size_t mp = ns_pad(std::min(rows, cols)), np = ns_pad(std::max(rows, cols));
  return (ns_align((size_t)batch * NS_NORM_PARTS * 8) + NS_ARRIVED * 4 + (size_t)batch * 4 * (3 * mp * np + 3 * mp * mp)) / 4;
}

static long long ns_tiles(int edge, int rows_a, int rows_b, bool symmetric) {
  const long long ta = (rows_a + edge - 1) / edge, tb = (rows_b + edge - 1) / edge;
  return symmetric ? ta * (ta + 1) / 2 : ta * tb;
}
template <int S, int G, int KIND, typename T>
static hipError_t ns_launch_small(hipStream_t s, dim3 grid, const NsParams& p, const NsProduct& q) {
  static bool allowed = false;
  hipError_t e = pp_allow_lds((const void*)ns_product_kernel<S, G, KIND, T>, NsSmall<S, G>::LDS, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((ns_product_kernel<S, G, KIND, T>), grid, dim3(256 * G), (NsSmall<S, G>::LDS), s, p, q);
  return hipGetLastError();
}
// One product of every matrix of the batch.  64 wide tiles where two workgroups a CU hold them all, with the contraction dealt to four groups
// of waves where there is a workgroup a CU, else to two (one matrix of 1024 x 1024: four groups 197 us, two 213, one 247).  More of
// them would take a second round: then 128 wide ones, in two groups where each CU has one (2048 x 2048: 64 wide 904 us, 128 wide in two groups
// 791, in one 1071; six of 1024 x 1024: 64 wide 581, 531, 649), in one where each CU has more (24 of 768 x 2048: 1721, 1587, 1542);
// for a symmetric product with a few more of them than CUs, which would take twice the time of one, 64 wide again (four of 1344 x 1792, 264
// tiles: 1028 us against 1153; 325 tiles of 3200 x 3200: 2608 against 2448; but of the products with X, 272 tiles of four of 2100 x
// 410: 236 against 221).  256 wide tiles where they fill the chip (24 of 1024 x 4096: 128 wide 4.4 ms, 3.7), and for
// the products with X, which write most, from 144 on (160 of 2500 x 4000: 1720 -> 1481 us; 128 of eight of 1024 x 1024: 736 -> 762;
// symmetric, 144 of 24 of 768 x 2048: 1542 -> 1692).  No tile is more than twice as wide as a matrix is high.
template <int KIND, typename T>
static hipError_t ns_product(hipStream_t s, const NsParams& p, NsProduct q, int batch) {
  const bool symmetric = KIND == NS_PLAIN || KIND == NS_POLY;
  auto tiles = [&](int edge) { return ns_tiles(edge, q.rows_a, q.rows_b, symmetric) * batch; };
  int edge = 128;
  if (tiles(64) <= 512 || q.rows_a <= 64) edge = 64;
  else if (q.rows_a > 128 && tiles(256) >= (symmetric ? 192 : 144)) edge = 256;
  else if (symmetric && tiles(128) > 256 && tiles(128) <= 300) edge = 64;
  q.tiles = (int)ns_tiles(edge, q.rows_a, q.rows_b, symmetric);
  q.tiles_b = symmetric ? 0 : (q.rows_b + edge - 1) / edge;
  // A workgroup a CU at most, whose share of the contraction costs it what the sums of the other shares cost the one that adds them up: n K-tiles at
  // 0.09 us against k_tiles / n shares at 0.27 us.  (64 x 4096: 116 -> 68 us, 64 x 16384 362 -> 96, 410 x 2100 176 -> 153, 50257 x
  // 128 1155 -> 255; 512 x 512 is as before.)  `parts` has the place of a matrix X.
  if (q.parts && edge == 64) {
    const long long room = (long long)p.mp * p.np / (q.tiles * 4096ll), share = std::max(8, (int)std::sqrt(3.0 * q.k_tiles));
    const int want = (int)std::min({256ll / (q.tiles * batch), q.k_tiles / share, room});
    if (want > 1) {
      q.per = (q.k_tiles + want - 1) / want;
      q.splits = (q.k_tiles + q.per - 1) / q.per;
    }
  }
  const dim3 grid((unsigned)(q.tiles * batch * q.splits));
  if (q.splits > 1) return ns_launch_small<1, 4, KIND, T>(s, grid, p, q);
  if (edge == 256) {
    static bool allowed = false;
    hipError_t e = pp_allow_lds((const void*)ns_product_pp_kernel<KIND, T>, PP_LDS, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((ns_product_pp_kernel<KIND, T>), grid, dim3(512), PP_LDS, s, p, q);
    return hipGetLastError();
  }
  if (edge == 128) return q.tiles * batch <= 256 ? ns_launch_small<2, 2, KIND, T>(s, grid, p, q) : ns_launch_small<2, 1, KIND, T>(s, grid, p, q);
  return q.tiles * batch <= 256 && q.k_tiles >= 8 ? ns_launch_small<1, 4, KIND, T>(s, grid, p, q) : ns_launch_small<1, 2, KIND, T>(s, grid, p, q);
}

template <typename T>
static hipError_t ns_run(hipStream_t s, NsParams& p, int batch, int steps) {
  if (p.mp == 64 && p.np <= NS_ALONE_COLS) {
    static bool allowed = false;
    hipError_t e = pp_allow_lds((const void*)ns_alone_kernel<T>, NS_ALONE_LDS, allowed);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(ns_alone_kernel<T>, dim3(batch), dim3(64 * NS_ALONE_WAVES), NS_ALONE_LDS, s, p, steps);
    return hipGetLastError();
  }
  hipLaunchKernelGGL(ns_norm_kernel<T>, dim3(p.parts, batch), dim3(256), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(ns_start_kernel<T>, dim3(p.mp / 64 * (p.np / 64), batch), dim3(256), 0, s, p);
  e = hipGetLastError();
  const bool pairs = p.np >= 2 * p.mp || p.mp == 64;       // two steps with X once (see above); below, a pair is no less work, but for small matrices fewer launches
  for (int i = 0, half = 0; i < steps && e == hipSuccess; half ^= 1) {
    const bool two = pairs && i + 1 < steps;
    auto product = [&](auto kind, const char* l, const char* r, char* out) {
      NsProduct q;
      memset(&q, 0, sizeof q);
      q.a = l; q.b = r; q.rows_a = q.rows_b = p.mp; q.k_tiles = (l == p.x ? p.np : p.mp) / 32; q.out = out;
      q.splits = 1;
      if (l == p.x) q.parts = reinterpret_cast<double*>(p.xt[1 - half]);    // free until X is written
      if (e == hipSuccess) e = ns_product<decltype(kind)::value, float>(s, p, q, batch);
    };
    constexpr std::integral_constant<int, NS_PLAIN> plain{};
    constexpr std::integral_constant<int, NS_POLY> poly{};
    product(plain, p.x, p.x, p.gram);                      // A
    const char* by = p.gram;
    if (e == hipSuccess && p.mp == NsChain::M) {
      hipLaunchKernelGGL(ns_chain_kernel, dim3(batch), dim3(NsChain::THREADS), 2 * NsChain::BYTES, s, p.gram, (int)two);
      e = hipGetLastError();
    } else {
      product(poly, p.gram, p.gram, p.c);                  // C
      by = p.c;
    }
    if (two && p.mp != NsChain::M) {
      product(plain, p.c, p.gram, p.t);                    // C A
      product(plain, p.t, p.c, p.gram);                    // A' = C A C
      product(poly, p.gram, p.gram, p.t);                  // C'
      product(plain, p.t, p.c, p.gram);                    // C' C
      by = p.gram;
    }
    i += two ? 2 : 1;
    if (e != hipSuccess) break;
    NsProduct q;
    memset(&q, 0, sizeof q);
    q.splits = 1;
    q.a = by; q.b = p.xt[half]; q.rows_a = p.mp; q.rows_b = p.np; q.k_tiles = p.mp / 32; q.out = p.x; q.out_t = p.xt[1 - half];
    e = i < steps ? ns_product<NS_NEXT, float>(s, p, q, batch) : ns_product<NS_LAST, T>(s, p, q, batch);
  }
  return e;
}

hipError_t launch_orthogonalize(hipStream_t s, int dtype, const OrthogonalizeDesc& d) {
  NsParams p;
  memset(&p, 0, sizeof p);
  p.rows = d.rows; p.cols = d.cols; p.tall = d.rows > d.cols;
  p.m = std::min(d.rows, d.cols); p.n = std::max(d.rows, d.cols); p.mp = ns_pad(p.m); p.np = ns_pad(p.n);
  p.g = d.g; p.ldg = d.ldg; p.sg = d.sg; p.mom = d.momentum; p.mu = d.mu; p.nesterov = d.nesterov;
  p.o = d.o; p.ldo = d.ldo; p.so = d.so; p.scale = d.scale; p.eps = d.eps;
  p.parts = std::min({NS_NORM_PARTS, (p.rows + 3) / 4, std::max(16, 2048 / d.batch)});
  const size_t big = (size_t)d.batch * p.mp * p.np * 4, small = (size_t)d.batch * p.mp * p.mp * 4;
  char* at = reinterpret_cast<char*>(d.scratch);
  p.sums = reinterpret_cast<double*>(at); at += ns_align((size_t)d.batch * NS_NORM_PARTS * 8);
  p.arrived = reinterpret_cast<unsigned*>(at); at += NS_ARRIVED * 4;
  p.x = at; at += big;
  p.xt[0] = at; at += big;
  p.xt[1] = at; at += big;
  p.gram = at; at += small;
  p.c = at; at += small;
  p.t = at;
  return dtype == 1 ? ns_run<bf16_t>(s, p, d.batch, d.steps) : ns_run<float>(s, p, d.batch, d.steps);
}

}  // namespace ouro
