// Orthogonalised updates: X = U / (|U|_F + eps), then steps of X <- a X + (b A + c A^2) X with A = X X^T, which drive the singular
// values of U towards 1 and leave its singular vectors (Newton-Schulz with the quintic whose coefficients are below).  U is the
// gradient or its momentum.
//
// The products run on fp16 matrix instructions with every operand as a sum of two fp16 numbers, high + low (22 bits of
// mantissa): x y = xh yh + xh yl + xl yh with fp32 accumulation.  One fp16 (or bf16) number is not enough: a step multiplies small singular
// values by a, five steps by 485, and with them the rounding noise of X: with 16 strong directions over noise of 1e-4 one
// fp16 number gives an error of 4.5e-2, bf16 0.37, the two halves 8e-6 and fp32 arithmetic 5e-6 (random matrices: 1.4e-3, 1.1e-2,
// 2.6e-7, 1.7e-7).  All entries of X, A and the polynomial are below 5 in magnitude (|X|_2 <= 1.2); they are stored times 2^12, so that
// the low halves of ordinary entries (1 / sqrt(rows cols)) stay above fp16's smallest normal number.
//
// All three products are of the form A B^T with the contraction contiguous in both: X X^T; the square of the symmetric A; and
// (the polynomial, symmetric) times X^T, for which X is kept in both layouts.  Of the two symmetric results only the
// tiles on and below the diagonal are formed and stored twice.  Matrices are the smaller dimension times the larger, padded with zeros
// to whole multiples of 64: zero rows and columns stay zero in every step.
#include "common.h"
#include "unaligned.h"

#include <algorithm>

namespace ouro {

typedef _Float16 half_t;
typedef __attribute__((ext_vector_type(4))) _Float16 half4;
typedef __attribute__((ext_vector_type(8))) _Float16 half8;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((address_space(3))) void ns_lds_void;

constexpr float NS_A = 3.4445f, NS_B = -4.7750f, NS_C = 2.0315f;
constexpr float NS_SCALE = 4096.f, NS_DOWN = 1.f / 4096.f;
constexpr int NS_NORM_PARTS = 256;                         // most partial sums of squares of a matrix

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
  char *x, *xt[2], *gram, *poly;                           // split matrices, batch after batch
};

// ------------------------------------------------------------------------- norm, momentum
// What is orthogonalised, from the gradient and the updated momentum.
__device__ __forceinline__ float ns_update(const NsParams& p, float g, float mom) { return !p.mom ? g : p.nesterov ? fmaf(p.mu, mom, g) : mom; }

// Momentum, and the sum of squares in 64 bits: no gradient is too large or too small for it.
template <typename T>
__global__ __launch_bounds__(256) void ns_norm_kernel(NsParams p) {
  __shared__ double part[4];
  const int b = blockIdx.y;
  const T* g = reinterpret_cast<const T*>(p.g) + b * p.sg;
  float* mom = p.mom ? p.mom + b * p.sg : nullptr;
  double sum = 0;
  for (int r = blockIdx.x; r < p.rows; r += p.parts)
    for (int c = threadIdx.x; c < p.cols; c += 256) {
      const size_t at = r * p.ldg + c;
      const float x = to_f32(g[at]);
      float m = 0.f;
      if (mom) mom[at] = m = fmaf(p.mu, mom[at], x);
      const double u = ns_update(p, x, m);
      sum += u * u;
    }
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
  __syncthreads();
  if (threadIdx.x == 0) p.sums[(size_t)b * p.parts + blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

// X and its transpose, split and padded, from 64 x 64 tiles.
template <typename T>
__global__ __launch_bounds__(256) void ns_start_kernel(NsParams p) {
  __shared__ float tile[64][65];
  __shared__ double part[4];
  const int tid = threadIdx.x, b = blockIdx.y, tiles_n = p.np / 64;
  const int r0 = blockIdx.x / tiles_n * 64, c0 = blockIdx.x % tiles_n * 64;    // of X
  double sum = tid < p.parts ? p.sums[(size_t)b * p.parts + tid] : 0;
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
  if ((tid & 63) == 0) part[tid >> 6] = sum;
  __syncthreads();
  const double inv = NS_SCALE / (sqrt((part[0] + part[1]) + (part[2] + part[3])) + p.eps);    // in 64 bits as the sum
  const T* g = reinterpret_cast<const T*>(p.g) + b * p.sg;
  const float* mom = p.mom ? p.mom + b * p.sg : nullptr;
  const int i0 = p.tall ? c0 : r0, j0 = p.tall ? r0 : c0;                      // of the caller's matrix
  for (int k = tid; k < 64 * 64; k += 256) {
    const int i = k >> 6, j = k & 63;
    float u = 0.f;
    if (i0 + i < p.rows && j0 + j < p.cols) {
      const size_t at = (i0 + i) * p.ldg + j0 + j;
      u = (float)(ns_update(p, to_f32(g[at]), mom ? mom[at] : 0.f) * inv);
    }
    if (p.tall) tile[j][i] = u;
    else tile[i][j] = u;
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
enum { NS_GRAM = 0, NS_POLY = 1, NS_NEXT = 2, NS_LAST = 3 };
struct NsProduct {
  const char* a; const char* b;                            // split [rows_a][32 k_tiles], [rows_b][32 k_tiles], batch after batch
  int rows_a, rows_b, k_tiles;
  int tiles_b;                                             // tiles along rows_b; symmetric results: 0
  int tiles;                                               // of one matrix
  const char* xt;                                          // NEXT, LAST: X^T
  char* out; char* out_t;                                  // GRAM, POLY: the result; NEXT: X and X^T
};

__device__ __forceinline__ void ns_request(const void* base, int bytes, char* dst, uint32_t voff, uint32_t k) {
  auto rs = __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, bytes, 0x00020000);
  __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (ns_lds_void*)dst, 16, voff, k, 0, 0);
}

// 64 S x 64 S tiles, four waves of 32 S x 32 S each.  A K-tile is 32 of the contraction: 128-byte rows of high and low halves in LDS, two
// stages, 16-byte chunk c of a row at c ^ swizzle(row).
template <int S, int KIND, typename T>
__global__ __launch_bounds__(256) void ns_product_kernel(NsParams p, NsProduct q) {
  constexpr int ROWS = 64 * S, STAGE = 2 * ROWS * 128;
  extern __shared__ char ns_lds[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = blockIdx.x / q.tiles, t = blockIdx.x - b * q.tiles;
  int ti, tj;
  if (q.tiles_b) { ti = t / q.tiles_b; tj = t - ti * q.tiles_b; }
  else {                                                   // row ti of the triangle begins at ti (ti + 1) / 2
    ti = (int)((sqrtf(8.f * t + 1.f) - 1.f) * 0.5f);
    while (ti * (ti + 1) / 2 > t) --ti;
    while ((ti + 1) * (ti + 2) / 2 <= t) ++ti;
    tj = t - ti * (ti + 1) / 2;
  }
  const int m0 = ti * ROWS, n0 = tj * ROWS, ld = q.k_tiles * 128;
  const int bytes_a = q.rows_a * ld, bytes_b = q.rows_b * ld;
  const char* A = q.a + (size_t)b * bytes_a;
  const char* B = q.b + (size_t)b * bytes_b;
  auto swizzle = [](int row) { return (row ^ (row >> 3)) & 7; };
  auto request = [&](int kt) __attribute__((always_inline)) {
    char* dst = ns_lds + (kt & 1) * STAGE;
#pragma unroll
    for (int i = 0; i < 2 * S; ++i) {                      // 8 rows a request
      const int row = (wave * 2 * S + i) * 8 + (lane >> 3);
      const uint32_t off = (uint32_t)(((lane & 7) ^ swizzle(row)) << 4);
      ns_request(A, bytes_a, dst + (wave * 2 * S + i) * 1024, (uint32_t)(m0 + row) * ld + off, kt * 128);
      ns_request(B, bytes_b, dst + ROWS * 128 + (wave * 2 * S + i) * 1024, (uint32_t)(n0 + row) * ld + off, kt * 128);
    }
  };
  f32x16_t acc[S][S];
#pragma unroll
  for (int i = 0; i < S; ++i)
#pragma unroll
    for (int j = 0; j < S; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
  const int wm = (wave >> 1) * 32 * S, wn = (wave & 1) * 32 * S;
  request(0);
  for (int kt = 0; kt < q.k_tiles; ++kt) {
    __syncthreads();                                       // K-tile kt has arrived, and nobody reads the other stage
    if (kt + 1 < q.k_tiles) request(kt + 1);
    const char* st = ns_lds + (kt & 1) * STAGE;
    half8 fa[S][4], fb[S][4];                              // chunks: high 0-15, high 16-31, low 0-15, low 16-31
#pragma unroll
    for (int i = 0; i < S; ++i)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const int ra = wm + 32 * i + (lane & 31), rb = wn + 32 * i + (lane & 31), ch = 2 * c + (lane >> 5);
        fa[i][c] = *reinterpret_cast<const half8*>(st + ra * 128 + ((ch ^ swizzle(ra)) << 4));
        fb[i][c] = *reinterpret_cast<const half8*>(st + ROWS * 128 + rb * 128 + ((ch ^ swizzle(rb)) << 4));
      }
#pragma unroll
    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int j = 0; j < S; ++j) {
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[i][ks], fb[j][ks], acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[i][ks], fb[j][2 + ks], acc[i][j], 0, 0, 0);
          acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[i][2 + ks], fb[j][ks], acc[i][j], 0, 0, 0);
        }
  }
  // ---- epilogue: a lane holds four neighbouring rows (m) of one column (n)
  const int cols_t = q.rows_a;                             // row length of what is stored with m contiguous
  const size_t mat = (size_t)b * q.rows_a * q.rows_b * 4;
#pragma unroll
  for (int i = 0; i < S; ++i)
#pragma unroll
    for (int j = 0; j < S; ++j) {
      const int n = n0 + wn + 32 * j + (lane & 31);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int m = m0 + wm + 32 * i + 8 * r + 4 * (lane >> 5);
        if (m >= q.rows_a || n >= q.rows_b) continue;
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * r + e] * NS_DOWN;
        if (KIND != NS_GRAM) {
          // POLY: A itself, symmetric; NEXT, LAST: X^T
          const char* old = (KIND == NS_POLY ? q.a : q.xt) + mat + ns_at(n, m, cols_t);
          const half4 hi = *reinterpret_cast<const half4*>(old), lo = *reinterpret_cast<const half4*>(old + 64);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = (float)hi[e] + (float)lo[e];
            v[e] = KIND == NS_POLY ? fmaf(NS_C, v[e], NS_B * x) : fmaf(NS_A, x, v[e]);
          }
        }
        if (KIND == NS_LAST) {
          T* o = reinterpret_cast<T*>(p.o) + b * p.so;
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (m + e < p.m && n < p.n) o[p.tall ? n * p.ldo + m + e : (m + e) * p.ldo + n] = from_f32<T>(v[e] * (p.scale * NS_DOWN));
          continue;
        }
        half4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          half_t h, l;
          ns_split(v[e], h, l);
          hi[e] = h; lo[e] = l;
        }
        char* at = (KIND == NS_NEXT ? q.out_t : q.out) + mat + ns_at(n, m, cols_t);
        *reinterpret_cast<half4*>(at) = hi;
        *reinterpret_cast<half4*>(at + 64) = lo;
        if (KIND != NS_NEXT && ti == tj) continue;         // a tile on the diagonal holds both of each pair
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          char* d = q.out + mat + ns_at(m + e, n, q.rows_b);
          *reinterpret_cast<half_t*>(d) = hi[e];
          *reinterpret_cast<half_t*>(d + 64) = lo[e];
        }
      }
    }
}

// ---------------------------------------------------------------------------------- host
static int ns_pad(int x) { return (x + 63) / 64 * 64; }
static size_t ns_align(size_t bytes) { return (bytes + 255) / 256 * 256; }
size_t orthogonalize_scratch_floats(int batch, int rows, int cols) {
  const size_t mp = ns_pad(std::min(rows, cols)), np = ns_pad(std::max(rows, cols));
  return (ns_align((size_t)batch * NS_NORM_PARTS * 8) + (size_t)batch * 4 * (3 * mp * np + 2 * mp * mp)) / 4;
}

template <int S, int KIND, typename T>
static hipError_t ns_product(hipStream_t s, const NsParams& p, NsProduct q, int batch) {
  constexpr int ROWS = 64 * S;
  const int ta = (q.rows_a + ROWS - 1) / ROWS, tb = (q.rows_b + ROWS - 1) / ROWS;
  const bool symmetric = KIND == NS_GRAM || KIND == NS_POLY;
  q.tiles_b = symmetric ? 0 : tb;
  q.tiles = symmetric ? ta * (ta + 1) / 2 : ta * tb;
  hipLaunchKernelGGL((ns_product_kernel<S, KIND, T>), dim3((unsigned)(q.tiles * batch)), dim3(256), 2 * 2 * ROWS * 128, s, p, q);
  return hipGetLastError();
}

template <typename T, int S>
static hipError_t ns_run(hipStream_t s, NsParams& p, int batch, int steps) {
  hipLaunchKernelGGL(ns_norm_kernel<T>, dim3(p.parts, batch), dim3(256), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(ns_start_kernel<T>, dim3(p.mp / 64 * (p.np / 64), batch), dim3(256), 0, s, p);
  e = hipGetLastError();
  for (int i = 0; i < steps && e == hipSuccess; ++i) {
    NsProduct q;
    memset(&q, 0, sizeof q);
    q.a = q.b = p.x; q.rows_a = q.rows_b = p.mp; q.k_tiles = p.np / 32; q.out = p.gram;
    e = ns_product<S, NS_GRAM, float>(s, p, q, batch);
    if (e != hipSuccess) break;
    q.a = q.b = p.gram; q.k_tiles = p.mp / 32; q.out = p.poly;
    e = ns_product<S, NS_POLY, float>(s, p, q, batch);
    if (e != hipSuccess) break;
    q.a = p.poly; q.b = q.xt = p.xt[i & 1]; q.rows_b = p.np; q.out = p.x; q.out_t = p.xt[1 - (i & 1)];
    e = i + 1 < steps ? ns_product<S, NS_NEXT, float>(s, p, q, batch) : ns_product<S, NS_LAST, T>(s, p, q, batch);
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
  p.parts = std::min({NS_NORM_PARTS, p.rows, std::max(16, 2048 / d.batch)});
  const size_t big = (size_t)d.batch * p.mp * p.np * 4, small = (size_t)d.batch * p.mp * p.mp * 4;
  char* at = reinterpret_cast<char*>(d.scratch);
  p.sums = reinterpret_cast<double*>(at); at += ns_align((size_t)d.batch * NS_NORM_PARTS * 8);
  p.x = at; at += big;
  p.xt[0] = at; at += big;
  p.xt[1] = at; at += big;
  p.gram = at; at += small;
  p.poly = at;
  return dtype == 1 ? ns_run<bf16_t, 1>(s, p, d.batch, d.steps) : ns_run<float, 1>(s, p, d.batch, d.steps);
}

}  // namespace ouro
