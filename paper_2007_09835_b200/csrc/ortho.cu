// Orthogonalised updates: Newton-Schulz products of a layer's gradient, and the optimiser step around them.
//
// With A = X X^T every step multiplies X by p(A) = a + b A + c A A, and the next A is p(A) A p(A): all of them polynomials in the
// first A, which commute and are symmetric.  So a few steps are taken on the small n x n matrices (n the shorter side, l the longer)
//     G = X X^T;   P_1 = p_1(G), G <- P_1 G P_1, P_2 = p_2(G), ..;   Q = .. P_2 P_1;   X <- Q X
// which reads X twice for up to three steps instead of twice a step, and of a symmetric product only the tiles on and under the
// diagonal are computed.  Squaring X loses the small singular values s where s^2 falls under the rounding of G; with 22 bits of G and at
// most three steps to a run (which enlarge by at most 41 = 3.4445^3) little is lost: directions against 64 bits, of |O|, and fp32 products beside
// them: noise of 64 x 576 6.9e-6 and 1.7e-6, 4096 x 8192 3.4e-5 and 7.2e-6; singular values as 1/i^2, 512 x 1024, 4.1e-5 and 2.5e-5; two
// directions only, 2000 x 3000, 3.5e-4 and 1.3e-4.  (Five steps in one run give NaN.)
// Values enter the tensor cores as fp16 parts, v = hi + lo (22 bits), products as hi hi + hi lo + lo hi with fp32 sums.  fp16's 11 bits
// against bf16's 8, and a bf16 gradient is its own hi part.  (The X before the last steps without its lo part, for a result in bf16,
// left 1.0e-3 of |O| beside that result's own rounding of 1.7e-3; it saved 3 to 16 %.)  Matrices are held times a power of two (2^14,
// 2^10 for P and Q) so that lo parts stay normal numbers.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdint>
#include <cstring>
#include <initializer_list>

#include "pdl.cuh"
#include "rt3d.h"
#include "rt3d_internal.h"
#include "umma_common.cuh"

namespace rt3d {

CUresult encode_tiled(CUtensorMap* map, CUtensorMapDataType type, cuuint32_t rank, void* data, const cuuint64_t* dims, const cuuint64_t* strides,
                      const cuuint32_t* box, const cuuint32_t* steps, CUtensorMapSwizzle swizzle);      // api.cu

namespace {

constexpr int kNormBlocks = 512;
constexpr int kMostSteps = 16, kRuns = kMostSteps;
// Up to this side the small matrices' products are steps of one launch.  A side of 512 against twice the length, five steps, us: as launches 154,
// as steps 145; 768: 187 and 176; 1024: 215 and 214; 1280: 280 and 285.
constexpr int kFusedSide = 1024;
// Where X is short as well, everything is, with runs of one step, which need the fewest products in a row, as long as X's tiles of
// 128 x 64 are one round of the SMs.  us, in runs of two and three and this way: side 64: 512 long 77 and 66, 768 79 and 74, 1024 79 and 82;
// side 256: 512 99 and 80, 768 102 and 100, 1024 102 and 107; side 512: 1024 145 and 134, 2048 149 and 168; side 768: 768 171 and 146,
// 1536 176 and 171 (144 tiles); side 896: 1344 190 and 174, 1536 191 and 211 (168 tiles); side 1024: 1024 199 and 172, 1280 207 and 218
// (160 tiles), 1536 208 and 226.
inline bool everything_fused(int n, int l, int sms) {
  return n <= kFusedSide && (l <= 768 || (l <= 2 * n && l <= 1536 && ceil_div(n, 128) * ceil_div(l, 64) <= sms));
}
constexpr float kXScale = 16384.f, kGScale = 16384.f, kPScale = 1024.f;        // what X, G and T, P and Q are held times

__device__ __forceinline__ float value_of(const float* p) { return *p; }
__device__ __forceinline__ float value_of(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// ------------------------------------------------------------------------------------------------ the matrix X of the first run
// The matrix whose direction is wanted: a plain one, or the one of an optimiser step, whose momentum is brought up to date when
// it is read first.
template <typename T>
struct Source {
  const T* g;
  long long pitch;
  float* momentum;         // nullptr: g itself
  const uint8_t* mask;
  float mu;
  int nesterov;
};
// Four neighbours of a row from column j on, those from `n` on zero.  kVec: all pointers allow wide accesses there.
template <typename T, bool kVec>
__device__ __forceinline__ void load4(const T* p, int n, float (&v)[4]) {
  if (kVec) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *reinterpret_cast<const float4*>(p);
      v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
    } else {
      const uint2 a = *reinterpret_cast<const uint2*>(p);
      v[0] = __uint_as_float(a.x << 16); v[1] = __uint_as_float(a.x & 0xffff0000u);
      v[2] = __uint_as_float(a.y << 16); v[3] = __uint_as_float(a.y & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = e < n ? value_of(p + e) : 0.f;
  }
}
// Four neighbours of the source: what they are made of, loaded, and then the values; the first kernel writes the momentum.
template <typename T, bool kVec>
struct Quad {
  float g[4], m[4];
  uint32_t keep;
  __device__ __forceinline__ void load(const Source<T>& s, long long g_at, long long at, int n) {
    load4<T, kVec>(s.g + g_at, n, g);
    keep = 0x01010101u;
    if (!s.momentum) return;
    load4<float, kVec>(s.momentum + at, n, m);
    if (!s.mask) return;
    if constexpr (kVec) {
      keep = *reinterpret_cast<const uint32_t*>(s.mask + at);
    } else {
      keep = 0;
      for (int e = 0; e < 4 && e < n; ++e) keep |= uint32_t(s.mask[at + e]) << (8 * e);
    }
  }
  template <bool kFirst>
  __device__ __forceinline__ void values(const Source<T>& s, long long at, int n, float (&v)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = g[e];
    if (!s.momentum) return;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const bool on = (keep >> (8 * e)) & 0xffu;
      if (kFirst) m[e] = on ? fmaf(s.mu, m[e], v[e]) : 0.f;
      v[e] = !on ? 0.f : s.nesterov ? fmaf(s.mu, m[e], v[e]) : m[e];
    }
    if (kFirst) {
      if constexpr (kVec) *reinterpret_cast<float4*>(s.momentum + at) = make_float4(m[0], m[1], m[2], m[3]);
      else
        for (int e = 0; e < 4 && e < n; ++e) s.momentum[at + e] = m[e];
    }
  }
};

// Sums of squares of the blocks' shares, in 64 bits: neither overflow nor the order of a long sum matters.  Four quads of a thread are
// on their way at a time; kFlat: rows without gaps, whose places need no division.
template <typename T, bool kVec, bool kFlat>
__global__ void __launch_bounds__(256)
square_sums_kernel(Source<T> s, int m, int k, double* __restrict__ sums) {
  pdl_entry();
  __shared__ double part[8];
  const unsigned quads = unsigned(k + 3) / 4;
  const long long total = kFlat ? (long long)m * k / 4 : (long long)m * quads;
  constexpr long long kStep = (long long)kNormBlocks * 256;
  double sum = 0.0;
  for (long long first = blockIdx.x * 256 + threadIdx.x; first < total; first += 4 * kStep) {
    Quad<T, kVec> quad[4];
    long long at[4];
    int n[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const long long idx = first + q * kStep;
      n[q] = 0;
      if (idx >= total) continue;
      if (kFlat) {
        at[q] = idx * 4; n[q] = 4;
        quad[q].load(s, at[q], at[q], 4);
      } else {
        const int i = total >> 32 ? int(idx / quads) : int(unsigned(idx) / quads), j = int(idx - (long long)i * quads) * 4;
        at[q] = (long long)i * k + j; n[q] = k - j;
        quad[q].load(s, (long long)i * s.pitch + j, at[q], n[q]);
      }
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if (n[q] == 0) continue;
      float v[4];
      quad[q].template values<true>(s, at[q], n[q], v);
#pragma unroll
      for (int e = 0; e < 4; ++e) sum += double(v[e]) * v[e];
    }
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += part[w];
    sums[blockIdx.x] = sum;
  }
}

// Two values at a time: a conversion of one takes as long as one of two, on a pipe of 16 lanes a clock.
__device__ __forceinline__ void split_half2(float x, float y, __half2& hi, __half2& lo) {
  hi = __floats2half2_rn(x, y);
  const float2 back = __half22float2(hi);
  lo = __floats2half2_rn(x - back.x, y - back.y);
}
__device__ __forceinline__ void split_half(float v, __half& hi, __half& lo) {
  hi = __float2half_rn(v);
  lo = __float2half_rn(v - __half2float(hi));
}

// The steps as the device needs them: how many each run takes, and their coefficients.
struct RunSteps {
  int runs;
  uint8_t steps[kRuns];
  float abc[kMostSteps][3];
};

// The matrix of run r is F_r times what is held.  F_0 is the source over its norm and eps, of which a power of two is taken here,
// which rounds nothing but what falls under fp16.  `size` bounds the matrix's singular values through the steps (|p| of a step is at most
// |a| + |b| s^2 + |c| s^4 there, and no step leaves more than 1.9): where a run leaves less than one, because eps is more than the norm or
// because its steps shrink, the next run's matrix is held times the power of two that brings that bound next to one, so that no
// gradient and no step takes the bits of the values under fp16's.
// factors[r]: F_r^2, for G; factors[kRuns + r]: F_r / F_(r + 1), for X.
__device__ void write_factors(double f, double size, const RunSteps& steps, float* __restrict__ factors) {
  int step = 0;
  for (int r = 0; r < steps.runs; ++r) {
    for (int i = 0; i < steps.steps[r]; ++i, ++step) {
      const double square = size * size;
      size *= fabs(steps.abc[step][0]) + square * (fabs(steps.abc[step][1]) + square * fabs(steps.abc[step][2]));
      if (size > 1.9) size = 1.9;
    }
    double next = 1.0;
    if (r + 1 < steps.runs && size > 0.0 && size < 1.0) next = scalbn(1.0, ilogb(size) + 1);
    factors[r] = float(f * f);
    factors[kRuns + r] = float(f / next);
    f = next;
  }
}

// Blocks take 32 x 128 places; turned where there are more rows than columns, through shared memory.
template <typename T, bool kVec>
__global__ void __launch_bounds__(256)
split_kernel(Source<T> s, int m, int k, const double* __restrict__ sums, double eps, int turned, __half* __restrict__ hi,
             __half* __restrict__ lo, long long x_pitch, const __grid_constant__ RunSteps steps, float* __restrict__ factors,
             unsigned* __restrict__ arrived) {
  pdl_entry();
  __shared__ double part[8];
  __shared__ float tile[32][133];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int cols = (k + 127) / 128;
  const int i0 = int(blockIdx.x / cols) * 32, j0 = int(blockIdx.x % cols) * 128, j = j0 + lane * 4;
  Quad<T, kVec> quad[4];                                         // on their way while the norm is worked out
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int i = i0 + p * 8 + warp;
    if (i < m && j < k) quad[p].load(s, (long long)i * s.pitch + j, (long long)i * k + j, k - j);
  }
  double sum = sums[threadIdx.x] + sums[threadIdx.x + 256];
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  __shared__ float scale_s[2];                                   // powers of two, whose product may leave the range of 32 bits
  if (blockIdx.x == 0 && threadIdx.x < kRuns) arrived[threadIdx.x] = 0;
  if (threadIdx.x == 0) {                                        // one thread: 64-bit roots and exponents are slow
    sum = part[0];
    for (int w = 1; w < 8; ++w) sum += part[w];
    const double norm = sqrt(sum);
    const bool number = norm > 0.0 && norm < 1e300;              // one that is none makes everything NaN
    const int e = number ? -ilogb(norm) - 1 : 0, up = e + 14, first = up / 2;  // norm * 2^e in [1/2, 1)
    const double power = scalbn(1.0, e);
    scale_s[0] = scalbnf(1.f, first); scale_s[1] = scalbnf(1.f, up - first);
    if (blockIdx.x == 0)
      write_factors(number ? 1.0 / ((norm + eps) * power) : norm == 0.0 ? 1.0 : __longlong_as_double(0x7fffffffffffffffll),
                    number ? norm / (norm + eps) : 0.0, steps, factors);
  }
  __syncthreads();
  const float scale0 = scale_s[0], scale1 = scale_s[1];
  static_assert(kXScale == 16384.f, "2^14");
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const int r = p * 8 + warp, i = i0 + r;
    if (i >= m || j >= k) continue;
    float v[4];
    quad[p].template values<false>(s, 0, 0, v);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = v[e] * scale0 * scale1;
    if (turned) {
#pragma unroll
      for (int e = 0; e < 4; ++e) tile[r][lane * 4 + e] = v[e];
      continue;
    }
    __half2 h2[2], l2[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) split_half2(v[2 * e], v[2 * e + 1], h2[e], l2[e]);
    const __half *h = reinterpret_cast<const __half*>(h2), *l = reinterpret_cast<const __half*>(l2);
    __half *to = hi + i * x_pitch + j, *lo_to = lo + i * x_pitch + j;
    if (j + 4 <= k) {                                            // the pitch is a multiple of 8
      *reinterpret_cast<uint2*>(to) = *reinterpret_cast<const uint2*>(h2);
      if (lo) *reinterpret_cast<uint2*>(lo_to) = *reinterpret_cast<const uint2*>(l2);
    } else {
      for (int e = 0; e < 4 && j + e < k; ++e) {
        to[e] = h[e];
        if (lo) lo_to[e] = l[e];
      }
    }
  }
  if (!turned) return;
  __syncthreads();
  for (int c = warp; c < 128; c += 8) {
    const int j = j0 + c, i = i0 + lane;
    if (j >= k || i >= m) continue;
    __half h, l;
    split_half(tile[lane][c], h, l);
    hi[j * x_pitch + i] = h;
    if (lo) lo[j * x_pitch + i] = l;
  }
}

// ------------------------------------------------------------------------------------------------------------- products
constexpr int kTile = 128;                           // rows of a tile
constexpr uint32_t kRowsBytes = kTile * 128;         // of 128 x 64 fp16
constexpr int kProductThreads = 320;                 // producer, issuer, eight warps for the results
constexpr int kMostProblems = 16;                    // of one launch
constexpr int kMostCluster = 16;

// Tiles of 128 x kCols: a stage holds 64 of the sum of up to four operands (hi and lo of A and B), as many as the launch's products have.
template <int kCols>
struct Stage {
  static constexpr uint32_t kColsBytes = kCols * 128, kRingBytes = 3 * (2 * kRowsBytes + 2 * kColsBytes);
  // results on their way out (128 x 64): hi and lo
  static constexpr uint32_t kOutAt = kRingBytes, kAllBytes = kCols == 64 ? kOutAt + 2 * kRowsBytes : kRingBytes;
  // columns of an accumulator: with both parts of B side by side, hi hi and hi lo are one product where kCols is 64 (120 clocks for 16 of
  // the sum of all three parts, 168 one after another)
  static constexpr int kAcc = 128;
  static constexpr int kSumsAt = 2 * kAcc, kTmemCols = 512;            // behind the accumulators: kCols of sums so far (a power of two in all)
};
// The tensor core cuts addends off as it adds, which in sums of one sign (the diagonal of X X^T) goes one way: an accumulator takes 512 of a
// sum, then the other one goes on while its values are added, rounded to nearest, to those before it, which lie in tensor memory too.
// An update's direction against 64 bits, of |O|, with one accumulator to a sum and with this: 4096 x 8192 2.0e-4 and 3.4e-5, 1500 x 1500
// 9.5e-5 and 4.4e-5, 130 x 2^18 2.2e-4 and 5.9e-6 (of noise), for 2 to 5 % of the time; segments of 256 halve the larger ones again for 2 % more.
constexpr int kSegment = 8;                          // chunks of 64, at most

enum { kOutParts = 0, kOutDirection = 1, kOutUpdate = 2 };

// One product C = A B from A's rows and B^T's (K-major operands), or B's own (X, the last product of a run).  Of a symmetric matrix only
// the 128 x 128 blocks on and under the diagonal are there: what a row has above them is the transpose of a block under the diagonal and
// enters the product as such.
// The descriptors of a matrix in the workspace, hi and lo: boxes of 64 columns by 128 and by 64 rows.  One table of them serves all
// products of a call: the few descriptors that a launch uses stay in their cache, where a set for every product made each
// copy wait for its own (2000 clocks of a step's 6500).
enum { kX0, kX1, kG0, kG1, kP0, kP1, kT, kQ0, kQ1, kMatrices };
struct Maps { CUtensorMap rows128[2], rows64[2]; };
struct Problem {
  int out;                                           // what becomes of C = alpha * factor * sum + diag I + beta D
  float alpha, beta, diag;
  const float* factor;                               // nullptr: 1
  const __half *d_hi, *d_lo;                         // D, or nullptr
  __half *c_hi, *c_lo;                               // kOutParts
  long long pitch;                                   // of C and D
  int parts;                                         // 1: hi hi; 2: hi hi + lo hi; 3: and hi lo
  int same;                                          // A and B are the same matrix: a tile on the diagonal loads it once
  int a, b, c;                                       // the matrices; c < 0: none of them
  int a_under, b_under;                              // A, B is symmetric and lies on and under the diagonal only
  int b_rows;                                        // B's own rows
  int symmetric;                                     // so is C: tiles on and under the diagonal
  int chunks;
  int segment, segments;                             // chunks of an accumulator, accumulators of a sum (of the largest share of one)
  int tiles_m, n_tiles;
  int rows, cols;                                    // what of C exists (symmetric: all of the tiles)
};
// Products of a launch: the problems [first[s], first[s + 1]) of a step run beside one another, every step after the one before.
template <int kProblems>
struct Steps {
  Problem p[kProblems];
  int first[kProblems + 1];
};
template <int kProblems>
struct ProductArgs {
  Maps m[kMatrices];
  Steps<kProblems> steps;
  int n_steps, splits;
  int ring;                                          // stages
  uint32_t b_at, stage_bytes;
  int one_cluster;                                   // the grid is a cluster, which is what steps wait through
  unsigned* arrived;                                 // else: CTAs that have reached the ends of steps, all together
  // results outside
  int turned;                                        // C is written as its transpose
  __nv_bfloat16* bf;
  float* w;
  const uint8_t* mask;
  float keep_share, step;
  long long w_pitch;
  int32_t* err;
};

template <int kCols>
constexpr uint32_t kProductSmem = Stage<kCols>::kAllBytes + 1024 + sizeof(Barriers) + sizeof(Steps<kMostProblems>) + 16;

// fp16 x fp16 -> fp32, M = 128; A K-major or transposed, B K-major or its own rows.
template <int kCols>
__device__ __forceinline__ uint32_t instr_desc_f16(bool a_turned, bool b_rows) {
  return (1u << 4) | (a_turned ? 1u << 15 : 0u) | (b_rows ? 1u << 16 : 0u) | (uint32_t(kCols >> 3) << 17) | (uint32_t(kTile >> 4) << 24);
}
// Rows along the sum: 64 columns (128 bytes, swizzled) by rows of the sum; 8 rows 1024 bytes apart, 64 columns 8192.
__device__ __forceinline__ uint64_t smem_desc_rows(uint32_t addr) {
  return uint64_t((addr & 0x3FFFFu) >> 4) | uint64_t(8192 >> 4) << 16 | uint64_t(1024 >> 4) << 32 | uint64_t(1) << 46 | uint64_t(2) << 61;
}

struct TileAt { int problem, i, j; };
// Whether chunk c of the rows `at`.. of a symmetric matrix lies above the blocks that are there.
__device__ __forceinline__ bool above(int under, int c, int at) { return under && c * 64 >= (at / kTile + 1) * kTile; }
template <int kCols, int kProblems>
__device__ __forceinline__ TileAt tile_at(const Steps<kProblems>& a, int s, int item) {
  TileAt t;
  t.problem = a.first[s];
  while (item >= a.p[t.problem].n_tiles) item -= a.p[t.problem++].n_tiles;
  const Problem& p = a.p[t.problem];
  if (p.symmetric) {                                 // tiles before row i: w i (i + 1) / 2 with w of kCols to a row of 128
    constexpr int w = kTile / kCols;
    t.i = int((sqrtf(8.f * float(item) / w + 1.f) - 1.f) * 0.5f);
    while (w * t.i * (t.i + 1) / 2 > item) --t.i;
    while (w * (t.i + 1) * (t.i + 2) / 2 <= item) ++t.i;
    t.j = item - w * t.i * (t.i + 1) / 2;
  } else {
    t.j = item / p.tiles_m;                          // rows of tiles fastest: neighbours share B
    t.i = item - t.j * p.tiles_m;
  }
  return t;
}
// 16 values of D, which are there before the product is.
struct Addend {
  uint4 hi[2], lo[2];
  __device__ __forceinline__ void load(const Problem& p, long long at) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      hi[q] = __ldcg(reinterpret_cast<const uint4*>(p.d_hi + at + 8 * q));
      lo[q] = __ldcg(reinterpret_cast<const uint4*>(p.d_lo + at + 8 * q));
    }
  }
};

// 16 columns from c0 on of this thread's row of a tile.
template <int kCols, int kProblems>
__device__ __forceinline__ void finish16(const ProductArgs<kProblems>& a, const Problem& p, const TileAt& t, int row, int c0, float (&v)[16], float alpha,
                                         const Addend& d) {
  const int i = t.i * kTile + row, j = t.j * kCols + c0;
#pragma unroll
  for (int e = 0; e < 16; ++e) v[e] *= alpha;
  if (p.out == kOutParts) {
    if (p.symmetric) {                               // small matrices, whole tiles
      if (p.d_hi) {
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const uint4 h = d.hi[q], l = d.lo[q];
          const __half2 *hh = reinterpret_cast<const __half2*>(&h), *ll = reinterpret_cast<const __half2*>(&l);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 x = __half22float2(hh[e]), y = __half22float2(ll[e]);
            v[8 * q + 2 * e] += p.beta * (x.x + y.x); v[8 * q + 2 * e + 1] += p.beta * (x.y + y.y);
          }
        }
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (i == j + e) v[e] += p.diag;
      }
    } else if (i >= p.rows) {
      return;
    }
    __half2 h[8], l[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) split_half2(v[2 * e], v[2 * e + 1], h[e], l[e]);
    const long long at = i * p.pitch + j;
#pragma unroll
    for (int q = 0; q < 2; ++q)
      if (j + 8 * q < p.cols) {                      // the pitch is a multiple of 8: what lies behind the last column is padding
        *reinterpret_cast<uint4*>(p.c_hi + at + 8 * q) = reinterpret_cast<const uint4*>(h)[q];
        *reinterpret_cast<uint4*>(p.c_lo + at + 8 * q) = reinterpret_cast<const uint4*>(l)[q];
      }
    return;
  }
  if (i >= p.rows) return;
  const int n = p.cols - j;
  if (p.out == kOutDirection) {
    if (a.turned) {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e < n) a.bf[(j + e) * a.w_pitch + i] = __float2bfloat16_rn(v[e]);
      return;
    }
    __nv_bfloat16* to = a.bf + i * a.w_pitch + j;
    if (n >= 16 && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
      uint32_t o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
        o[e] = *reinterpret_cast<const uint32_t*>(&b);
      }
      reinterpret_cast<uint4*>(to)[0] = make_uint4(o[0], o[1], o[2], o[3]);
      reinterpret_cast<uint4*>(to)[1] = make_uint4(o[4], o[5], o[6], o[7]);
    } else {
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (e < n) to[e] = __float2bfloat16_rn(v[e]);
    }
    return;
  }
  if (a.turned) {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e < n) {
        const long long at = (j + e) * a.w_pitch + i;
        a.w[at] = !a.mask || a.mask[at] ? fmaf(-a.step, v[e], a.keep_share * a.w[at]) : 0.f;
      }
    return;
  }
  const long long at = i * a.w_pitch + j;
  float* to = a.w + at;
  if (n >= 16 && ((reinterpret_cast<uintptr_t>(to) | (a.mask ? reinterpret_cast<uintptr_t>(a.mask + at) : 0)) & 15) == 0) {
    uint4 keep = make_uint4(0x01010101u, 0x01010101u, 0x01010101u, 0x01010101u);
    if (a.mask) keep = *reinterpret_cast<const uint4*>(a.mask + at);
    const uint32_t k4[4] = {keep.x, keep.y, keep.z, keep.w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float4 x = reinterpret_cast<const float4*>(to)[q];
      x.x = k4[q] & 0xffu ? fmaf(-a.step, v[4 * q], a.keep_share * x.x) : 0.f;
      x.y = k4[q] & 0xff00u ? fmaf(-a.step, v[4 * q + 1], a.keep_share * x.y) : 0.f;
      x.z = k4[q] & 0xff0000u ? fmaf(-a.step, v[4 * q + 2], a.keep_share * x.z) : 0.f;
      x.w = k4[q] & 0xff000000u ? fmaf(-a.step, v[4 * q + 3], a.keep_share * x.w) : 0.f;
      reinterpret_cast<float4*>(to)[q] = x;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e)
      if (e < n) to[e] = !a.mask || a.mask[at + e] ? fmaf(-a.step, v[e], a.keep_share * to[e]) : 0.f;
  }
}

__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, uint32_t src, int c0, int c1) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];"
               ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, const uint4& v) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]));
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void add_sums(uint32_t sums, uint32_t (&r)[32]) {
  uint32_t so_far[32];
  tmem_ld32(sums, so_far);
#pragma unroll
  for (int e = 0; e < 32; ++e) r[e] = __float_as_uint(__uint_as_float(so_far[e]) + __uint_as_float(r[e]));
}
// A thread has the columns half * 32 .. + 31 of every 64 of its row.  Adds the accumulators of `segments` segments to its sums; `n` counts
// the accumulators.
template <int kCols>
__device__ __forceinline__ bool drain(const Problem& p, uint32_t lanes, int half, int segments, uint32_t& n, int lane, Barriers* bars, int32_t* err) {
  typedef Stage<kCols> S;
  for (int g = 0; g < segments; ++g, ++n) {
    const uint32_t buf = n & 1u;
    if (!mbar_wait_warp(smem_u32(&bars->tmem_full[buf]), (n >> 1) & 1u, bars, err, 4)) return false;
    tc_fence_after();
#pragma unroll 1
    for (int c = half * 32; c < kCols; c += 64) {
      uint32_t r[32];
      __syncwarp();
      tmem_ld_acc(lanes + buf * S::kAcc + c, true, kCols == 64 && p.parts == 3 ? uint32_t(kCols) : 0u, r);
      if (g) add_sums(lanes + S::kSumsAt + c, r);
      tmem_st32(lanes + S::kSumsAt + c, r);
    }
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&bars->tmem_empty[buf]));
  }
  return true;
}

// The parts of a tile of 128 x 64 through shared memory and out in whole rows; D comes the same way, to the places its thread then
// writes.  (16-byte accesses of a row each, which touch 32 lines, kept the SM's load and store unit busy for 2000 clocks of a
// step's 8000.)  Called by all 256 threads.
template <int kCols>
__device__ __forceinline__ void finish_staged(const Problem& p, const Maps* maps, const TileAt& t, uint32_t taddr, uint32_t sums, int row, int half, float alpha, uint32_t base,
                                              uint32_t tmem_full, uint32_t full_parity, uint32_t d_parity, Barriers* bars, int32_t* err) {
  typedef Stage<kCols> S;
  const bool leader = threadIdx.x == 64, add = p.d_hi != nullptr;
  const uint32_t out = base + S::kOutAt, d_bar = smem_u32(&bars->full[kMaxStages - 1]);
  if (leader) {
    tma_store_wait_read_0();
    if (add) {
      mbar_expect_tx(d_bar, 2 * kRowsBytes);
      for (int q = 0; q < 2; ++q) tma_load_2d(out + q * kRowsBytes, &maps[p.a].rows128[q], d_bar, t.j * kCols, t.i * kTile);
    }
  }
  bool ok = mbar_wait_warp(tmem_full, full_parity, bars, err, 4);
  tc_fence_after();
  epilogue_bar_sync(256);                            // the leader has waited for the last tile's way out
  if (add) ok = mbar_wait_warp(d_bar, d_parity, bars, err, 6) && ok;
  if (ok) {
    const uint32_t line = out + row * 128;
    const int diagonal = p.symmetric ? t.i * kTile + row - t.j * kCols - half * 32 : -1;        // of this row's columns
    uint32_t r[32];
    __syncwarp();
    tmem_ld_acc(taddr + half * 32, true, p.parts == 3 ? uint32_t(kCols) : 0u, r);
    if (sums) add_sums(sums + half * 32, r);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t at = line + (((half * 4 + u) ^ (row & 7)) << 4);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = alpha * __uint_as_float(r[8 * u + e]);
      if (add) {
        const uint4 dh = lds128(at), dl = lds128(at + kRowsBytes);
        const __half2 *hh = reinterpret_cast<const __half2*>(&dh), *ll = reinterpret_cast<const __half2*>(&dl);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 x = __half22float2(hh[e]), y = __half22float2(ll[e]);
          v[2 * e] += p.beta * (x.x + y.x); v[2 * e + 1] += p.beta * (x.y + y.y);
        }
        if ((diagonal >> 3) == u) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] += (diagonal & 7) == e ? p.diag : 0.f;
        }
      }
      __half2 h[4], l[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) split_half2(v[2 * e], v[2 * e + 1], h[e], l[e]);
      sts128(at, *reinterpret_cast<const uint4*>(h));
      sts128(at + kRowsBytes, *reinterpret_cast<const uint4*>(l));
    }
  }
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  epilogue_bar_sync(256);
  if (leader && ok) {
    for (int q = 0; q < 2; ++q) tma_store_2d(&maps[p.c].rows128[q], out + q * kRowsBytes, t.j * kCols, t.i * kTile);
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
  }
}

// All CTAs of a cooperative grid have ended the step: `target` arrivals in all.  Bounded like every wait here.
__device__ __forceinline__ void grid_barrier(unsigned* arrived, unsigned target, Barriers* bars, int32_t* err) {
  __threadfence();
  __syncwarp();
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    atomicAdd(arrived, 1u);
    const long long start = clock64();
    unsigned seen;
    for (;;) {
      asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(seen) : "l"(arrived) : "memory");
      if (seen >= target) break;
      if (clock64() - start > bars->wait_limit) {
        bars->abort_flag = 1;
        atomicCAS(err, 0, 5);
        break;
      }
    }
    __threadfence();
  }
  __syncthreads();
}

// TMA fills a ring of stages, one thread issues the products of a stage's parts, eight warps take results from the two accumulators:
// one tile after another in a CTA.  With splits (one step, one tile to a cluster), the CTAs of a cluster share the sum and add
// their parts up through one another's shared memory, 128 / splits columns each: the products X X^T have few tiles and long sums.
// With several steps, the CTAs wait for one another between them, as one cluster or as a cooperative grid: a step on small matrices is
// shorter than a launch.
template <int kCols, int kProblems>
__global__ void __launch_bounds__(kProductThreads, 1)
product_kernel(const __grid_constant__ ProductArgs<kProblems> a) {
  typedef Stage<kCols> S;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  Barriers* bars = reinterpret_cast<Barriers*>(smem_raw + (base - smem_u32(smem_raw)) + S::kAllBytes);
  Steps<kProblems>& steps = *reinterpret_cast<Steps<kProblems>*>(bars + 1);
  const int warp = uniform(int(threadIdx.x >> 5)), lane = threadIdx.x & 31;
  const int split = a.splits > 1 ? int(cluster_ctarank()) : 0;
  const int cta = int(blockIdx.x) / a.splits, n_ctas = int(gridDim.x) / a.splits;

  if (threadIdx.x == 0) {
    for (int s = 0; s < a.ring; ++s) { mbar_init(smem_u32(&bars->full[s]), 1); mbar_init(smem_u32(&bars->empty[s]), 1); }
    for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&bars->tmem_full[b]), 1); mbar_init(smem_u32(&bars->tmem_empty[b]), 8); }
    mbar_init(smem_u32(&bars->full[kMaxStages - 1]), 1);         // of D
    bars->abort_flag = 0;
    bars->wait_limit = kWaitCycles;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  // What is read from the parameters on first use makes every step wait: the steps go to shared memory, the descriptors to their cache.
  static_assert(sizeof(steps) % 4 == 0, "copied by words");
  for (int q = int(threadIdx.x); q < int(sizeof(steps) / 4); q += kProductThreads)
    reinterpret_cast<uint32_t*>(&steps)[q] = reinterpret_cast<const uint32_t*>(&a.steps)[q];
  if (warp >= 2)
    for (int q = int(threadIdx.x) - 64; q < (kProblems > 1 ? kMatrices * 4 : 0); q += kProductThreads - 64) tma_prefetch_map(&a.m[0].rows128[0] + q);
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&bars->tmem_base)), "r"(uint32_t(S::kTmemCols)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(uint32_t(bars->tmem_base));
  pdl_launch();
  pdl_wait();

  int stage = 0;                                     // of this role: the ring and the accumulators go on from step to step
  uint32_t phase = 0, n = 0, adds = 0;
  bool joined = false;
#pragma unroll 1
  for (int s = 0; s < a.n_steps; ++s) {
    int n_items = 0;
    for (int p = steps.first[s]; p < steps.first[s + 1]; ++p) n_items += steps.p[p].n_tiles;
    TileAt t0{0, 0, 0};                              // this CTA's first, found while the others end the last step
    if (cta < n_items) t0 = tile_at<kCols>(steps, s, cta);
    if (kProblems > 1 && s > 0) {
      // What the last step's bulk stores have written is what this one's copies read, in other CTAs.  The stores' completion makes the
      // values visible to the thread that waits for it, the barrier passes that on, and the fence puts the copies, which go through the
      // other proxy, behind it.
      if (threadIdx.x == 64) tma_store_wait_all();
      if (a.one_cluster) {                           // a release and an acquire of the cluster
        __syncwarp();
        cluster_sync_all();
      } else {
        grid_barrier(a.arrived, unsigned(s) * gridDim.x, bars, a.err);
        if (bars->abort_flag) break;                 // this CTA's steps end here; the others' waits run out
      }
      asm volatile("fence.proxy.async.global;" ::: "memory");
    }
    if (warp == 0) {
      // ---------------------------------------------------------------- loads
      // Lanes 0 to 3 copy A hi, A lo, B hi and B lo, lanes 4 to 7 the second 64 columns of those that come as transposes: a copy's
      // address, descriptor and coordinates are 200 clocks of one thread's time.
      const int q = lane & 1, h = lane >> 2;
      const bool of_b = lane & 2;
      bool ok = true;
      for (int item = cta; item < n_items && ok; item += n_ctas) {
        const TileAt t = item == cta ? t0 : tile_at<kCols>(steps, s, item);
        const Problem& p = steps.p[t.problem];
        const bool one = kCols == kTile && p.same && t.i == t.j;
        const int a_parts = p.parts >= 2 ? 2 : 1, b_parts = one ? 0 : p.parts == 3 ? 2 : 1;
        const uint32_t bytes = uint32_t(a_parts) * kRowsBytes + uint32_t(b_parts) * S::kColsBytes;
        const Maps& m = a.m[of_b ? p.b : p.a];
        const CUtensorMap *straight = of_b && kCols == 64 ? &m.rows64[q] : &m.rows128[q], *turned = &m.rows64[q];
        const uint32_t to = base + (of_b ? a.b_at + q * S::kColsBytes : q * kRowsBytes);
        const int at = of_b ? t.j * kCols : t.i * kTile, under = of_b ? p.b_under : p.a_under;
        const bool always = of_b && p.b_rows, mine = lane < 8 && q < (of_b ? b_parts : a_parts), wide = !of_b || kCols == kTile;
        const int c_last = p.chunks * (split + 1) / a.splits;
        for (int c = p.chunks * split / a.splits; c < c_last; ++c) {
          const uint32_t full = smem_u32(&bars->full[stage]);
          const bool is_turned = always || above(under, c, at);
          if (!mbar_wait_warp(smem_u32(&bars->empty[stage]), phase ^ 1u, bars, a.err, 1)) { ok = false; break; }
          if (lane == 0) mbar_expect_tx(full, bytes);
          __syncwarp();
          if (mine && h <= (is_turned && wide ? 1 : 0)) {
            if (is_turned) tma_load_2d(to + stage * a.stage_bytes + h * 8192, turned, full, at + 64 * h, c * 64);
            else tma_load_2d(to + stage * a.stage_bytes, straight, full, c * 64, at);
          }
          if (++stage == a.ring) { stage = 0; phase ^= 1u; }
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      // ---------------------------------------------------------------- products
      const bool elected = elect_one();
      bool ok = true;
      for (int item = cta; item < n_items && ok; item += n_ctas, ++n) {
        const TileAt t = item == cta ? t0 : tile_at<kCols>(steps, s, item);
        const Problem& p = steps.p[t.problem];
        const bool one = kCols == kTile && p.same && t.i == t.j;
        uint32_t buf = 0, d = 0;
        const int c_first = p.chunks * split / a.splits, c_last = p.chunks * (split + 1) / a.splits;
        for (int c = c_first, left = 0; c < c_last; ++c, --left) {
          const bool first = left == 0;              // of an accumulator
          if (first) {
            left = p.segment;
            if (c > c_first) {
              if (elected) umma_commit(smem_u32(&bars->tmem_full[buf]));
              ++n;
            }
            buf = n & 1u; d = tmem + buf * S::kAcc;
            if (!mbar_wait_warp(smem_u32(&bars->tmem_empty[buf]), ((n >> 1) & 1u) ^ 1u, bars, a.err, 2)) { ok = false; break; }
            tc_fence_after();
          }
          if (!mbar_wait_warp(smem_u32(&bars->full[stage]), phase, bars, a.err, 3)) { ok = false; break; }
          tc_fence_after();
          const uint32_t at = base + stage * a.stage_bytes, b_at = one ? at : at + a.b_at, b_lo_at = one ? at + kRowsBytes : b_at + S::kColsBytes;
          const bool a_turned = above(p.a_under, c, t.i * kTile), b_turned = p.b_rows || above(p.b_under, c, t.j * kCols);
          const uint32_t idesc = instr_desc_f16<kCols>(a_turned, b_turned);
          const uint64_t a_step = a_turned ? (16 * 128) >> 4 : 32 >> 4, b_step = b_turned ? (16 * 128) >> 4 : 32 >> 4;      // 16 of the sum
          const uint64_t a_hi = a_turned ? smem_desc_rows(at) : smem_desc_sw128(at);
          const uint64_t a_lo = a_turned ? smem_desc_rows(at + kRowsBytes) : smem_desc_sw128(at + kRowsBytes);
          const uint64_t b_hi = b_turned ? smem_desc_rows(b_at) : smem_desc_sw128(b_at);
          const uint64_t b_lo = b_turned ? smem_desc_rows(b_lo_at) : smem_desc_sw128(b_lo_at);
          if (elected) {
            const bool both = kCols == 64 && p.parts == 3;
            const uint32_t more = first ? 0u : 1u;
            if (both) {                              // hi hi and hi lo side by side
              const uint32_t wide = instr_desc_f16<128>(a_turned, b_turned);
#pragma unroll
              for (int k = 0; k < 4; ++k) umma_bf16(d, a_hi + a_step * k, b_hi + b_step * k, wide, k ? 1u : more);
            } else {
#pragma unroll
              for (int k = 0; k < 4; ++k) umma_bf16(d, a_hi + a_step * k, b_hi + b_step * k, idesc, k ? 1u : more);
              if (p.parts == 3)
#pragma unroll
                for (int k = 0; k < 4; ++k) umma_bf16(d, a_hi + a_step * k, b_lo + b_step * k, idesc, 1u);
            }
            if (p.parts >= 2)
#pragma unroll
              for (int k = 0; k < 4; ++k) umma_bf16(d, a_lo + a_step * k, b_hi + b_step * k, idesc, 1u);
            umma_commit(smem_u32(&bars->empty[stage]));
          }
          if (++stage == a.ring) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        if (elected) umma_commit(smem_u32(&bars->tmem_full[buf]));
      }
      __syncwarp();
    } else {
      // ---------------------------------------------------------------- results
      const int quad = warp & 3, half = (warp - 2) >> 2, row = quad * 32 + lane;
      for (int item = cta; item < n_items; item += n_ctas, ++n) {
        const TileAt t = item == cta ? t0 : tile_at<kCols>(steps, s, item);
        const Problem& p = steps.p[t.problem];
        const float alpha = p.factor ? p.alpha * __ldcg(p.factor) : p.alpha;
        const uint32_t lanes = tmem + (uint32_t(quad * 32) << 16);
        int segments = p.segments;
        if (a.splits > 1) segments = (p.chunks * (split + 1) / a.splits - p.chunks * split / a.splits + p.segment - 1) / p.segment;
        const bool drained = drain<kCols>(p, lanes, half, segments - 1, n, lane, bars, a.err);
        const uint32_t buf = n & 1u, at = lanes + buf * S::kAcc, sums = segments > 1 ? lanes + S::kSumsAt : 0u;
        Addend d;
        const long long d_at = (t.i * kTile + row) * p.pitch + t.j * kCols;
        if (kCols == 64 && p.out == kOutParts) {
          finish_staged<kCols>(p, a.m, t, at, sums, row, half, alpha, base, smem_u32(&bars->tmem_full[buf]), (n >> 1) & 1u, adds & 1u, bars, a.err);
          adds += p.d_hi != nullptr;
          tc_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(smem_u32(&bars->tmem_empty[buf]));
          continue;
        }
        if (!drained || !mbar_wait_warp(smem_u32(&bars->tmem_full[buf]), (n >> 1) & 1u, bars, a.err, 4)) break;
        tc_fence_after();
        if (a.splits > 1) {          // this CTA's only tile: its part goes where the stages were, which every product has read
          store_partial_row(at, kCols, true, reinterpret_cast<float*>(smem_raw + (base - smem_u32(smem_raw))) + row * kPartRow, half * 32, 64,
                            sums ? sums - at : 0u);
        } else {
#pragma unroll 1
          for (int u = 0; u < kCols / 32; ++u) {
            const int c0 = (u >> 1) * 64 + half * 32 + (u & 1) * 16;
            uint32_t r[16];
            if (p.d_hi) d.load(p, d_at + c0);
            __syncwarp();
            tmem_ld16(at + c0, r);
            float v[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] = __uint_as_float(r[e]);
            if (kCols == 64 && p.parts == 3) {
              tmem_ld16(at + kCols + c0, r);
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] += __uint_as_float(r[e]);
            }
            if (sums) {
              tmem_ld16(sums + c0, r);
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] += __uint_as_float(r[e]);
            }
            finish16<kCols>(a, p, t, row, c0, v, alpha, d);
          }
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->tmem_empty[buf]));
        if (a.splits > 1) {
          cluster_sync_all();
          joined = true;
          if (!bars->abort_flag) {
            constexpr int units = kCols / 16;
            const int u1 = units * (split + 1) / a.splits;
#pragma unroll 1
            for (int u = units * split / a.splits + half; u < u1; u += 2) {
              const uint32_t local = base + uint32_t(u * 16 * 128 + row * kPartRow) * 4u;
              float v[16] = {};
#pragma unroll 2
              for (int q = 0; q < a.splits; ++q) {
                const uint32_t remote = mapa_shared(local, uint32_t(q));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  float4 x;
                  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                               : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(remote + e * 2048u) : "memory");
                  v[4 * e] += x.x; v[4 * e + 1] += x.y; v[4 * e + 2] += x.z; v[4 * e + 3] += x.w;
                }
              }
              if (p.d_hi) d.load(p, d_at + u * 16);
              finish16<kCols>(a, p, t, row, u * 16, v, alpha, d);
            }
          }
        }
      }
    }
  }
  if (kCols == 64 && threadIdx.x == 64) tma_store_wait_all();
  if (a.splits > 1) {
    // the results' warps have waited once, the others not; and nobody leaves while its part is still being read
    __syncwarp();
    if (warp < 2 || !joined) cluster_sync_all();
    cluster_sync_all();
  }
  if (bars->abort_flag) {
    // give copies and products still in flight time to land before TMEM goes away
    const long long t0 = clock64();
    while (clock64() - t0 < 2000000ll) { }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(uint32_t(S::kTmemCols)) : "memory");
  }
}

// ----------------------------------------------------------------------------------------------------------------- host
constexpr double kMostOfRun = 50.0;                  // a run's P and Q, held times 2^10, stay in fp16
struct Plan {
  int steps;
  double eps;
  float abc[kMostSteps][3];
  double most[kMostSteps];                           // largest |p| of a step
};

// Largest |q(s)| over [0, top] of q = s (a + b s^2 + c s^4), and of p = a + b s^2 + c s^4: at the ends or where a derivative is zero.
void bounds_of(double a, double b, double c, double top, double* most_q, double* most_p) {
  double at[5] = {0.0, top, 0.0, 0.0, 0.0};
  int n = 2;
  auto add = [&](double square) {
    if (square > 0.0 && square < top * top) at[n++] = std::sqrt(square);
  };
  if (c != 0.0) {                                        // q' = a + 3 b t + 5 c t^2, t = s^2;  p' = b + 2 c t
    const double disc = 9.0 * b * b - 20.0 * a * c;
    if (disc >= 0.0) { add((-3.0 * b + std::sqrt(disc)) / (10.0 * c)); add((-3.0 * b - std::sqrt(disc)) / (10.0 * c)); }
    add(-b / (2.0 * c));
  } else if (b != 0.0) {
    add(-a / (3.0 * b));
  }
  *most_q = *most_p = 0.0;
  for (int i = 0; i < n; ++i) {
    const double t = at[i] * at[i], p = a + t * (b + t * c);
    *most_p = std::fmax(*most_p, std::fabs(p));
    *most_q = std::fmax(*most_q, std::fabs(at[i] * p));
  }
}

rt3d_status make_plan(const rt3d_ortho_params* p, Plan* plan) {
  static const float usual[3] = {3.4445f, -4.7750f, 2.0315f};
  plan->steps = p ? p->steps : 5;
  plan->eps = p ? p->eps : 1e-7f;
  if (plan->steps < 1 || plan->steps > kMostSteps || !(plan->eps > 0.0) || !std::isfinite(plan->eps)) return RT3D_ERR_INVALID_ARG;
  double top = 1.0;
  for (int i = 0; i < plan->steps; ++i) {
    for (int e = 0; e < 3; ++e) {
      plan->abc[i][e] = p && p->coefs ? p->coefs[3 * i + e] : usual[e];
      if (!std::isfinite(plan->abc[i][e])) return RT3D_ERR_INVALID_ARG;
    }
    double most_p;
    bounds_of(plan->abc[i][0], plan->abc[i][1], plan->abc[i][2], top, &top, &most_p);
    if (!(top <= 1.9) || !(most_p <= kMostOfRun)) return RT3D_ERR_UNSUPPORTED;
    plan->most[i] = most_p;
  }
  return RT3D_OK;
}


struct Matrix {                                      // hi and lo parts, row-major
  __half *hi, *lo;
  int rows, cols;
  long long pitch;
};
struct Workspace {
  double* sums;
  float* factors;
  unsigned* arrived;                                 // [kRuns], of the launches with several steps
  Matrix all[kMatrices];
};
int64_t workspace_of(int m, int k, char* base, Workspace* out) {
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    char* p = base + at;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  auto matrix = [&](int rows, int cols, int64_t pitch) {
    Matrix x;
    x.rows = rows; x.cols = cols; x.pitch = pitch;
    x.hi = reinterpret_cast<__half*>(take(rows * pitch * 2));
    x.lo = reinterpret_cast<__half*>(take(rows * pitch * 2));
    return x;
  };
  const int n = m < k ? m : k, l = m < k ? k : m, side = int(ceil_div64(n, kTile)) * kTile;
  Workspace w;
  w.sums = reinterpret_cast<double*>(take(kNormBlocks * 8));
  w.factors = reinterpret_cast<float*>(take(2 * kRuns * 4));
  w.arrived = reinterpret_cast<unsigned*>(take(kRuns * 4));
  for (int i = 0; i < kMatrices; ++i) w.all[i] = i <= kX1 ? matrix(n, l, ceil_div64(l, 8) * 8) : matrix(side, side, side);
  if (out) *out = w;
  return at;
}

rt3d_status launched(cudaError_t e) {
  if (e != cudaSuccess) return RT3D_ERR_CUDA;
  count_launches(1);
  return RT3D_OK;
}

// Products as they are listed, and how they are launched: a step of its own each, or several steps in one launch.
struct Runner {
  DeviceInfo dev;
  cudaStream_t st;
  const Workspace& ws;
  Maps maps[kMatrices];
  const Matrix& matrix(int id) const { return ws.all[id]; }

  static bool map_of(CUtensorMap* map, const __half* p, const Matrix& x, int box_rows) {
    const cuuint64_t dims[2] = {cuuint64_t(x.cols), cuuint64_t(x.rows)}, strides[1] = {cuuint64_t(x.pitch) * 2};
    const cuuint32_t box[2] = {64, cuuint32_t(box_rows)}, estr[2] = {1, 1};
    return encode_tiled(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<__half*>(p), dims, strides, box, estr, CU_TENSOR_MAP_SWIZZLE_128B) == CUDA_SUCCESS;
  }
  bool make_maps() {
    for (int i = 0; i < kMatrices; ++i) {
      const Matrix& x = ws.all[i];
      for (int q = 0; q < 2; ++q)
        if (!map_of(&maps[i].rows128[q], q ? x.lo : x.hi, x, kTile) || !map_of(&maps[i].rows64[q], q ? x.lo : x.hi, x, 64)) return false;
    }
    return true;
  }

  // tiles of n x n on and under the diagonal: as wide as 128 rows need, the last row as wide as n
  static int tiles_under(int n, int cols) {
    const int rows = ceil_div(n, kTile), w = kTile / cols;
    return w * (rows - 1) * rows / 2 + (cols == kTile ? rows : ceil_div(n, cols));
  }
  // G = X X^T (of one or two parts)
  void gram(Problem* p, int x, int x_parts, int g, const float* factor, int cols) const {
    p->a = p->b = x; p->c = g;
    p->parts = x_parts == 2 ? 3 : 1; p->same = 1; p->symmetric = 1;
    p->chunks = ceil_div(matrix(x).cols, 64);
    p->n_tiles = tiles_under(matrix(x).rows, cols);
    p->factor = factor;
    p->alpha = kGScale / (kXScale * kXScale);
    out_parts(p, g);
  }
  // C = alpha L R of small symmetric matrices of which n x n exist
  void small(Problem* p, int n, int l, int r, int c, float alpha, int cols) const {
    p->a = l; p->b = r; p->c = c;
    p->parts = 3; p->symmetric = 1; p->a_under = p->b_under = 1;
    p->chunks = ceil_div(n, 64);
    p->n_tiles = tiles_under(n, cols);
    p->alpha = alpha;
    out_parts(p, c);
  }
  // P = a + b G + c G G
  void polynomial(Problem* p, int n, int g, int c, const float* abc, int cols) const {
    small(p, n, g, g, c, abc[2] * kPScale / (kGScale * kGScale), cols);
    p->same = 1;
    p->beta = abc[1] * kPScale / kGScale; p->diag = abc[0] * kPScale;
    p->d_hi = matrix(g).hi; p->d_lo = matrix(g).lo;
  }
  // alpha Q X; where it goes is the caller's to say
  void apply(Problem* p, int q, int x_id, int x_parts, const float* factor, int cols) const {
    const Matrix& x = matrix(x_id);
    p->a = q; p->b = x_id; p->c = -1;
    p->parts = x_parts == 2 ? 3 : 2; p->a_under = 1; p->b_rows = 1;
    p->chunks = ceil_div(x.rows, 64);
    p->tiles_m = ceil_div(x.rows, kTile); p->n_tiles = p->tiles_m * ceil_div(x.cols, cols);
    p->rows = x.rows; p->cols = x.cols;
    p->factor = factor; p->alpha = 1.f / kPScale;
  }
  void out_parts(Problem* p, int c) const {
    const Matrix& m = matrix(c);
    p->out = kOutParts; p->c = c; p->c_hi = m.hi; p->c_lo = m.lo; p->pitch = m.pitch;
    p->rows = m.rows; p->cols = m.cols;
  }

  // Clusters of `size` CTAs (up to 16, where 8 are portable) that the device holds at once.
  template <int kCols, int kProblems>
  static int clusters_at_once(int size) {
    static std::atomic<int> known[kMaxDevices][kMostCluster + 1];             // and one
    const int d = current_device_index();
    if (d < 0) return 0;
    int v = known[d][size].load();
    if (v == 0) {
      const auto kernel = product_kernel<kCols, kProblems>;
      int n = 0;
      LaunchSetup ls(dim3(unsigned(size)), dim3(kProductThreads), kProductSmem<kCols>, nullptr, unsigned(size));
      ls.cfg.numAttrs = 1;                                       // the cluster dimension alone
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kProductSmem<kCols>)) != cudaSuccess ||
          cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
          cudaOccupancyMaxActiveClusters(&n, kernel, &ls.cfg) != cudaSuccess) {
        cudaGetLastError();
        n = 0;
      }
      v = n + 1;
      known[d][size].store(v);
    }
    return v - 1;
  }

  template <int kCols, int kProblems>
  rt3d_status launch(ProductArgs<kProblems>& a, int grid, unsigned cluster, bool cooperative) const {
    const auto kernel = product_kernel<kCols, kProblems>;
    static std::atomic<bool> attr_done[kMaxDevices];
    const int d = current_device_index();
    if (d < 0) return RT3D_ERR_CUDA;
    if (!attr_done[d].load()) {
      if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kProductSmem<kCols>)) != cudaSuccess) return RT3D_ERR_CUDA;
      attr_done[d].store(true);
    }
    int a_parts = 1, b_parts = 1;
    for (int i = 0; i < a.steps.first[a.n_steps]; ++i) {
      if (a.steps.p[i].parts >= 2) a_parts = 2;
      if (a.steps.p[i].parts == 3) b_parts = 2;
    }
    for (int i = 0; i < a.steps.first[a.n_steps]; ++i) {           // segments as long as one another: one is added while the next one's products run
      Problem& p = a.steps.p[i];
      const int share = ceil_div(p.chunks, a.splits);
      p.segments = ceil_div(share, kSegment);
      p.segment = ceil_div(share, p.segments);
    }
    a.b_at = a_parts * kRowsBytes;
    a.stage_bytes = a.b_at + b_parts * Stage<kCols>::kColsBytes;
    a.ring = int(Stage<kCols>::kRingBytes / a.stage_bytes);
    if (a.ring > kMaxStages - 1) a.ring = kMaxStages - 1;                      // the last barrier is D's
    a.err = dev.err;
    std::memcpy(a.m, maps, sizeof(maps));
    LaunchSetup ls(dim3(unsigned(grid)), dim3(kProductThreads), kProductSmem<kCols>, st, cluster);
    if (cooperative) {
      ls.attr[0].id = cudaLaunchAttributeCooperative;
      ls.attr[0].val.cooperative = 1;
      ls.cfg.numAttrs = 1;
    }
    return launched(cudaLaunchKernelEx(&ls.cfg, kernel, a));
  }
  // One step of tiles of 128 x 128, the sums cut where there are few.
  rt3d_status run(ProductArgs<2>& a, int n_problems) const {
    int items = 0;
    for (int i = 0; i < n_problems; ++i) items += a.steps.p[i].n_tiles;
    a.steps.first[0] = 0; a.steps.first[1] = n_problems; a.n_steps = 1;
    // the largest cluster of which the device holds one for every tile, two chunks and more to a CTA
    a.splits = 1;
    if (2 * items <= dev.sm_count)
      for (int s = kMostCluster; s > 1 && a.splits == 1; --s)
        if (items * s <= dev.sm_count && a.steps.p[0].chunks >= 2 * s && clusters_at_once<kTile, 2>(s) >= items) a.splits = s;
    return launch<kTile>(a, a.splits > 1 ? items * a.splits : items < dev.sm_count ? items : dev.sm_count, unsigned(a.splits), false);
  }
};

// Steps of one launch, tiles of 128 x 64.
struct Fused {
  const Runner& r;
  ProductArgs<kMostProblems> a;
  int n_problems = 0;
  explicit Fused(const Runner& runner) : r(runner) { reset(); }
  void reset() {
    std::memset(&a, 0, sizeof(a));
    n_problems = 0;
  }
  Problem* add() { return &a.steps.p[n_problems++]; }
  void end_step() { a.steps.first[++a.n_steps] = n_problems; }
  // A cluster's wait takes 0.5 us, a grid's 1.5: a cluster's CTAs where going round more often than a grid would costs less than that
  // (a chunk of three products of 128 x 64: 700 clocks).
  rt3d_status run(unsigned* arrived) {
    const int side = Runner::clusters_at_once<64, kMostProblems>(kMostCluster) > 0 ? kMostCluster : 8;
    int most = 1, extra = 0;
    for (int s = 0; s < a.n_steps; ++s) {
      int items = 0;
      for (int p = a.steps.first[s]; p < a.steps.first[s + 1]; ++p) items += a.steps.p[p].n_tiles;
      most = items > most ? items : most;
      extra += (ceil_div(items, side) - ceil_div(items, r.dev.sm_count)) * a.steps.p[a.steps.first[s]].chunks;
    }
    a.splits = 1;
    a.one_cluster = extra * 700 <= a.n_steps * 1900;
    a.arrived = arrived;
    const int grid = a.one_cluster ? (most < side ? most : side) : most < r.dev.sm_count ? most : r.dev.sm_count;
    return r.launch<64>(a, grid, a.one_cluster ? unsigned(grid) : 1u, !a.one_cluster && a.n_steps > 1);
  }
};

// What becomes of the last product.
struct Result {
  int out, turned;
  __nv_bfloat16* bf;
  float* w;
  const uint8_t* mask;
  float keep_share, step;
  long long pitch;
};

// Steps of the run that begins at step `done`, at most `most`.
int run_steps(const Plan& plan, int done, int most) {
  int steps = 1;
  for (double p = plan.most[done]; steps < most && done + steps < plan.steps && (p *= plan.most[done + steps]) <= kMostOfRun;) ++steps;
  return steps;
}

template <typename T>
rt3d_status direction(const Source<T>& src, int m, int k, const Plan& plan, const Workspace& ws, const Result& res,
                      const DeviceInfo& dev, cudaStream_t st) {
  Runner r{dev, st, ws};
  if (!r.make_maps()) return RT3D_ERR_CUDA;
  const bool turned = m > k;
  const bool short_x = turned ? everything_fused(k, m, dev.sm_count) : everything_fused(m, k, dev.sm_count);
  uintptr_t bits = reinterpret_cast<uintptr_t>(src.g) | uintptr_t(src.pitch) * sizeof(T);       // 4 values at a time
  bool vec = k % 4 == 0 && bits % (4 * sizeof(T)) == 0;
  if (src.momentum) vec = vec && reinterpret_cast<uintptr_t>(src.momentum) % 16 == 0 && reinterpret_cast<uintptr_t>(src.mask) % 4 == 0;
  LaunchSetup l1(dim3(kNormBlocks), dim3(256), 0, st);
  rt3d_status s = launched(vec && src.pitch == k ? cudaLaunchKernelEx(&l1.cfg, square_sums_kernel<T, true, true>, src, m, k, ws.sums)
                           : vec                 ? cudaLaunchKernelEx(&l1.cfg, square_sums_kernel<T, true, false>, src, m, k, ws.sums)
                                                 : cudaLaunchKernelEx(&l1.cfg, square_sums_kernel<T, false, false>, src, m, k, ws.sums));
  if (s != RT3D_OK) return s;
  const Matrix* x = &ws.all[kX0];
  int parts = sizeof(T) == 2 && !src.momentum ? 1 : 2;           // a bf16 gradient is its own hi part
  __half* lo = parts == 2 ? x->lo : nullptr;
  RunSteps runs{};
  for (int done = 0; done < plan.steps; ++runs.runs) {
    runs.steps[runs.runs] = uint8_t(run_steps(plan, done, short_x ? 1 : runs.runs ? 3 : 2));
    done += runs.steps[runs.runs];
  }
  std::memcpy(runs.abc, plan.abc, sizeof(runs.abc));
  const long long blocks = ceil_div64(m, 32) * ceil_div64(k, 128);
  if (blocks >= (1ll << 31)) return RT3D_ERR_UNSUPPORTED;
  LaunchSetup l2(dim3(unsigned(blocks)), dim3(256), 0, st);
  s = launched(vec ? cudaLaunchKernelEx(&l2.cfg, split_kernel<T, true>, src, m, k, (const double*)ws.sums, plan.eps, int(turned), x->hi, lo, x->pitch, runs, ws.factors, ws.arrived)
                   : cudaLaunchKernelEx(&l2.cfg, split_kernel<T, false>, src, m, k, (const double*)ws.sums, plan.eps, int(turned), x->hi, lo, x->pitch, runs, ws.factors, ws.arrived));
  if (s != RT3D_OK) return s;
  const int n = turned ? k : m, n_fused = n <= kFusedSide;
  int launch_no = 0;
  ProductArgs<2> one;
  std::memset(&one, 0, sizeof(one));
  Fused chain(r);
  auto flush = [&]() -> rt3d_status {
    if (!chain.a.n_steps) return RT3D_OK;
    const rt3d_status e = chain.run(ws.arrived + launch_no++);
    chain.reset();
    return e;
  };
  int cur = kX0, other = kX1;
  for (int done = 0, run = 0; done < plan.steps; ++run) {
    const int steps = run_steps(plan, done, short_x ? 1 : run ? 3 : 2);
    int g = kG0, g2 = kG1, p = kP0, p2 = kP1, q = -1, q_next = kQ0;
    const int cols = n_fused ? 64 : kTile;
    if (short_x) {
      if (chain.n_problems + 3 > kMostProblems && (s = flush()) != RT3D_OK) return s;
      r.gram(chain.add(), cur, parts, g, ws.factors + run, cols);
      chain.end_step();
    } else {
      std::memset(&one, 0, sizeof(one));
      r.gram(&one.steps.p[0], cur, parts, g, ws.factors + run, kTile);
      if ((s = r.run(one, 1)) != RT3D_OK) return s;
    }
    // a step of one or two products
    auto products = [&](auto&& first_product, auto&& second_product, int count) -> rt3d_status {
      if (!n_fused) std::memset(&one, 0, sizeof(one));
      first_product(n_fused ? chain.add() : &one.steps.p[0]);
      if (count == 2) second_product(n_fused ? chain.add() : &one.steps.p[1]);
      if (!n_fused) return r.run(one, count);
      chain.end_step();
      return RT3D_OK;
    };
    for (int i = 0; i < steps; ++i) {
      const bool more = i + 1 < steps, has_q = q >= 0;
      auto make_p = [&](Problem* to) { r.polynomial(to, n, g, p, plan.abc[done + i], cols); };
      auto make_t = [&](Problem* to) { r.small(to, n, p, g, kT, kGScale / (kPScale * kGScale), cols); };         // T = P G
      auto make_q = [&](Problem* to) { r.small(to, n, p, q, q_next, 1.f / kPScale, cols); };                     // Q = P Q
      auto make_g = [&](Problem* to) { r.small(to, n, kT, p, g2, 1.f / kPScale, cols); };                        // G = T P
      if ((s = products(make_p, make_p, 1)) != RT3D_OK) return s;
      if (more || has_q) {
        s = more && has_q ? products(make_t, make_q, 2) : more ? products(make_t, make_t, 1) : products(make_q, make_q, 1);
        if (s != RT3D_OK) return s;
      }
      if (has_q) {
        q = q_next;
        q_next = q_next == kQ0 ? kQ1 : kQ0;
      }
      if (more) {
        if ((s = products(make_g, make_g, 1)) != RT3D_OK) return s;
        const int was = g; g = g2; g2 = was;
      }
      if (!has_q) { q = p; const int was = p; p = p2; p2 = was; }                                                // the first P is the first Q
    }
    done += steps;
    const bool last = done == plan.steps;
    if (!short_x) {
      if ((s = flush()) != RT3D_OK) return s;
      std::memset(&one, 0, sizeof(one));
    }
    Problem* c = short_x ? chain.add() : &one.steps.p[0];
    r.apply(c, q, cur, parts, ws.factors + kRuns + run, short_x ? cols : kTile);
    if (last) {
      c->out = res.out; c->alpha /= kXScale;
    } else {
      parts = 2;
      r.out_parts(c, other);
    }
    auto results = [&](auto& args) {
      args.turned = res.turned; args.bf = res.bf; args.w = res.w; args.mask = res.mask;
      args.keep_share = res.keep_share; args.step = res.step; args.w_pitch = res.pitch;
    };
    if (short_x) {
      chain.end_step();
      results(chain.a);
      if (last && (s = flush()) != RT3D_OK) return s;
    } else {
      results(one);
      if ((s = r.run(one, 1)) != RT3D_OK) return s;
    }
    const int was = cur; cur = other; other = was;
  }
  return RT3D_OK;
}

// Whether any two of a call's arrays share memory.
struct Area { const void* at; int64_t bytes; };
bool any_overlap(std::initializer_list<Area> areas) {
  for (const Area* a = areas.begin(); a != areas.end(); ++a)
    for (const Area* b = areas.begin(); b != a; ++b) {
      const uintptr_t a0 = reinterpret_cast<uintptr_t>(a->at), b0 = reinterpret_cast<uintptr_t>(b->at);
      if (a->at && b->at && a0 < b0 + uintptr_t(b->bytes) && b0 < a0 + uintptr_t(a->bytes)) return true;
    }
  return false;
}

rt3d_status check_call(const void* g, int dtype, int m, int k, void* workspace, int64_t bytes) {
  if (!g || !workspace || m < 1 || k < 1 || (dtype != RT3D_F32 && dtype != RT3D_BF16)) return RT3D_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(g) % (dtype == RT3D_BF16 ? 2 : 4) || reinterpret_cast<uintptr_t>(workspace) % 16) return RT3D_ERR_INVALID_ARG;
  const int64_t need = rt3d_ortho_workspace(m, k);
  if (need < 0) return RT3D_ERR_UNSUPPORTED;
  return bytes < need ? RT3D_ERR_WORKSPACE : RT3D_OK;
}


template <typename T>
rt3d_status orthogonalize(const T* g, int64_t pitch, int m, int k, const Plan& plan, __nv_bfloat16* out, int64_t out_pitch, char* base,
                          const DeviceInfo& dev, cudaStream_t st) {
  Workspace ws;
  workspace_of(m, k, base, &ws);
  const Result res{kOutDirection, m > k, out, nullptr, nullptr, 0.f, 0.f, (long long)out_pitch};
  return direction(Source<T>{g, pitch, nullptr, nullptr, 0.f, 0}, m, k, plan, ws, res, dev, st);
}

template <typename T>
rt3d_status update(float* w, float* momentum, const T* g, const uint8_t* mask, int m, int k, const rt3d_update_params& p, const Plan& plan,
                   char* base, const DeviceInfo& dev, cudaStream_t st) {
  Workspace ws;
  workspace_of(m, k, base, &ws);
  const Result res{kOutUpdate, m > k, nullptr, w, mask, float(1.0 - double(p.lr) * p.weight_decay), float(double(p.lr) * p.scale), k};
  return direction(Source<T>{g, k, momentum, mask, p.mu, p.nesterov}, m, k, plan, ws, res, dev, st);
}

}  // namespace
}  // namespace rt3d

using namespace rt3d;

extern "C" {

int64_t rt3d_ortho_workspace(int m, int k) {
  if (m < 1 || k < 1 || (m > 32768 && k > 32768) || m > (1 << 30) || k > (1 << 30)) return -1;
  return workspace_of(m, k, nullptr, nullptr);
}

rt3d_status rt3d_orthogonalize(const void* g, int dtype, int64_t g_pitch, int m, int k, const rt3d_ortho_params* p, void* out,
                               int64_t out_pitch, void* workspace, int64_t workspace_bytes, void* stream) {
  Plan plan;
  rt3d_status s = check_call(g, dtype, m, k, workspace, workspace_bytes);
  if (s != RT3D_OK) return s;
  if (!out || reinterpret_cast<uintptr_t>(out) % 2 || g_pitch < k || out_pitch < k) return RT3D_ERR_INVALID_ARG;
  const int64_t size = dtype == RT3D_BF16 ? 2 : 4;
  if (any_overlap({{g, ((m - 1) * g_pitch + k) * size}, {out, ((m - 1) * out_pitch + k) * 2}, {workspace, rt3d_ortho_workspace(m, k)}})) return RT3D_ERR_INVALID_ARG;
  if ((s = make_plan(p, &plan)) != RT3D_OK || plan_only()) return s;
  DeviceInfo dev;
  if ((s = current_device_info(&dev)) != RT3D_OK) return s;
  if (dev.cc_major != 10) return RT3D_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* base = static_cast<char*>(workspace);
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(out);
  return dtype == RT3D_BF16 ? orthogonalize(static_cast<const __nv_bfloat16*>(g), g_pitch, m, k, plan, o, out_pitch, base, dev, st)
                            : orthogonalize(static_cast<const float*>(g), g_pitch, m, k, plan, o, out_pitch, base, dev, st);
}

rt3d_status rt3d_ortho_update(float* w, float* momentum, const void* g, int dtype, const uint8_t* mask, int m, int k,
                              const rt3d_update_params* p, void* workspace, int64_t workspace_bytes, void* stream) {
  Plan plan;
  rt3d_status s = check_call(g, dtype, m, k, workspace, workspace_bytes);
  if (s != RT3D_OK) return s;
  if (!w || !momentum || !p || reinterpret_cast<uintptr_t>(w) % 4 || reinterpret_cast<uintptr_t>(momentum) % 4) return RT3D_ERR_INVALID_ARG;
  const int64_t count = int64_t(m) * k;
  if (any_overlap({{w, 4 * count}, {momentum, 4 * count}, {g, (dtype == RT3D_BF16 ? 2 : 4) * count}, {mask, count}, {workspace, rt3d_ortho_workspace(m, k)}}))
    return RT3D_ERR_INVALID_ARG;
  if (!std::isfinite(p->lr) || !std::isfinite(p->mu) || !std::isfinite(p->weight_decay) || !std::isfinite(p->scale)) return RT3D_ERR_INVALID_ARG;
  if ((s = make_plan(&p->ortho, &plan)) != RT3D_OK || plan_only()) return s;
  DeviceInfo dev;
  if ((s = current_device_info(&dev)) != RT3D_OK) return s;
  if (dev.cc_major != 10) return RT3D_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* base = static_cast<char*>(workspace);
  return dtype == RT3D_BF16 ? update(w, momentum, static_cast<const __nv_bfloat16*>(g), mask, m, k, *p, plan, base, dev, st)
                            : update(w, momentum, static_cast<const float*>(g), mask, m, k, *p, plan, base, dev, st);
}

}  // extern "C"
