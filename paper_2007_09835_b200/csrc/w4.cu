// 4-bit weights with group scales: quantisation, its inverse and the products with a few rows of activations.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "pdl.cuh"
#include "rt3d.h"
#include "rt3d_internal.h"
#include "umma_common.cuh"
#include "w4.cuh"

namespace rt3d {
namespace {

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}

__device__ __forceinline__ int shift_of(int e) { return 4 * ((e >> 1) + 4 * (e & 1)); }

// Scale, zero point and codes of a group as include/rt3d.h defines them.
struct Grid {
  float scale, zero;
  uint16_t bits;
};
__device__ __forceinline__ Grid grid_of(float low, float high, bool bad, bool zeros) {   // low <= 0 <= high
  Grid q;
  const float range = zeros ? __fdiv_rn(high - low, 15.f) : __fdiv_rn(fmaxf(high, -low), 7.f);
  q.bits = __bfloat16_as_ushort(__float2bfloat16_rn(range));
  q.scale = bf16_float(q.bits);
  if (bad || !(q.scale < __int_as_float(0x7f800000))) { q.bits = 0x7fffu; q.scale = 0.f; }
  q.zero = zeros && q.scale > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(-low, q.scale)), 0.f), 15.f) : 8.f;
  return q;
}
// The codes of eight values as a word.  A quotient decides between two codes only next to a half: elsewhere the product with the
// rounded reciprocal, off by less than 2^-19 of quotients up to 16, gives the same code, so eight values are divided only where one
// of them is that near (or the reciprocal out of range: a NaN).  Whole numbers are made by adding 1.5 2^23 (ties to even, as the
// rounding instruction, but on the pipe that has room) and read from the mantissa of 2^23 + code.
__device__ __forceinline__ uint32_t pack_codes(const float (&v)[8], const Grid& q, float inv) {
  constexpr float kWhole = 12582912.f;
  uint32_t word = 0;
  bool near = false;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = v[e] * inv, r = __fadd_rn(__fadd_rn(p, kWhole), -kWhole);
    near |= !(fabsf(p - r) < 0.49999f);
    word += (__float_as_uint(fminf(fmaxf(r + q.zero, 0.f), 15.f) + 8388608.f) - 0x4B000000u) << shift_of(e);
  }
  if (near) {
    word = 0;
#pragma unroll 1
    for (int e = 0; e < 8; ++e) {
      float x = v[0];
#pragma unroll
      for (int i = 1; i < 8; ++i) x = e == i ? v[i] : x;
      word |= uint32_t(fminf(fmaxf(rintf(__fdiv_rn(x, q.scale)) + q.zero, 0.f), 15.f)) << shift_of(e);
    }
  }
  return word;
}

// Eight values of a row in memory, those from `n` on zero; kVec: on a 16-byte boundary.
template <bool kVec>
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (kVec && n >= 8) {
    const float4 a = __ldg(reinterpret_cast<const float4*>(p)), b = __ldg(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? __ldg(p + e) : 0.f;
}
template <bool kVec>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int n, float (&v)[8]) {
  if (kVec && n >= 8) {
    const uint4 u = __ldg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = e < n ? __bfloat162float(p[e]) : 0.f;
}
template <bool kVec>
__device__ __forceinline__ void store4(float* p, int n, const float* v) {
  if (kVec && n >= 4) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < n) p[e] = v[e];
}
template <bool kVec>
__device__ __forceinline__ void store8(__nv_bfloat16* p, int n, const float (&v)[8]) {
  if (kVec && n >= 8) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * e], v[2 * e + 1]);
      w[e] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (e < n) p[e] = __float2bfloat16_rn(v[e]);
}

struct GridArgs {                    // of the two calls between 4-bit and plain weights
  uint4* codes;
  uint16_t* scales;
  uint8_t* zeros;
  long long pitch;
  int m, k, n_groups, k_blocks;
  long long chunks, total;           // what a warp takes, in a row of tiles and in all
};

// A warp takes 64 inputs of 16 filters, 128 where a group has as many: lane 4 g + t has 8 inputs of the filters g and g + 8 in each of
// the 32s, which are the words that it packs; four lanes make a group's extremes.  Read once, written in runs of 512 bytes.
// kGroup32: 32s in a group.
template <int kGroup32>
constexpr int kWarpBlocks = kGroup32 == 4 ? 2 : 1;          // blocks of 64 inputs that a warp takes
template <typename T, int kGroup32, bool kVec>
__global__ void __launch_bounds__(256)
w4_quantize_kernel(const T* __restrict__ w, const GridArgs a) {
  pdl_entry();
  const long long unit = ((long long)blockIdx.x * 256 + threadIdx.x) >> 5;
  if (unit >= a.total) return;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long long tile = unit / a.chunks;
  constexpr int kHalves = 2 * kWarpBlocks<kGroup32>;
  const int k0 = int(unit - tile * a.chunks) * (32 * kHalves);
  uint32_t words[2][kHalves];        // filter, 32 inputs
#pragma unroll
  for (int f = 0; f < 2; ++f) {
    const int i = int(tile) * 16 + g + 8 * f;
    const T* row = w + (long long)i * a.pitch;
    float v[kHalves][8], low[kHalves], high[kHalves];
    bool bad[kHalves];
    uint32_t filled = 0x88888888u;                   // the codes of values of zero
#pragma unroll
    for (int b = 0; b < kHalves; ++b) {
      const int at = k0 + b * 32 + t * 8;
      load8<kVec>(row + at, i < a.m ? a.k - at : 0, v[b]);
    }
#pragma unroll
    for (int b = 0; b < kHalves; ++b) {
      low[b] = high[b] = 0.f;
      bad[b] = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        low[b] = fminf(low[b], v[b][e]); high[b] = fmaxf(high[b], v[b][e]);
        bad[b] |= !(fabsf(v[b][e]) < __int_as_float(0x7f800000));
      }
#pragma unroll
      for (int o = 1; o <= 2; o *= 2) {
        low[b] = fminf(low[b], __shfl_xor_sync(0xffffffffu, low[b], o));
        high[b] = fmaxf(high[b], __shfl_xor_sync(0xffffffffu, high[b], o));
        bad[b] |= __shfl_xor_sync(0xffffffffu, int(bad[b]), o) != 0;
      }
    }
#pragma unroll
    for (int b = 0; b < kHalves; b += kGroup32) {
#pragma unroll
      for (int c = 1; c < kGroup32; ++c) {
        low[b] = fminf(low[b], low[b + c]); high[b] = fmaxf(high[b], high[b + c]); bad[b] |= bad[b + c];
      }
      const Grid q = grid_of(low[b], high[b], bad[b], a.zeros != nullptr);
      const int group = (k0 + b * 32) / (32 * kGroup32);
      if (t == 0 && group < a.n_groups) {
        const long long at = (tile * a.n_groups + group) * 16 + g + 8 * f;
        a.scales[at] = q.bits;
        if (a.zeros) a.zeros[at] = i < a.m ? uint8_t(q.zero) : 0;
      }
      // places that do not exist hold zeros; behind the last group they have its zero point
      const float inv = __fdiv_rn(1.f, q.scale);
      if (group < a.n_groups) filled = uint32_t(q.zero) * 0x11111111u;
#pragma unroll
      for (int c = 0; c < kGroup32; ++c) {
        words[f][b + c] = q.scale > 0.f ? pack_codes(v[b + c], q, inv) : filled;
      }
    }
  }
  uint4* dst = a.codes + (tile * a.k_blocks + k0 / 64) * 32 + lane;
#pragma unroll
  for (int b = 0; b < kHalves / 2; ++b)
    if (k0 / 64 + b < a.k_blocks) dst[b * 32] = make_uint4(words[0][2 * b], words[1][2 * b], words[0][2 * b + 1], words[1][2 * b + 1]);
}

template <typename T, int kGroup32, bool kVec>
__global__ void __launch_bounds__(256)
w4_unpack_kernel(T* __restrict__ w, const GridArgs a) {
  pdl_entry();
  const long long unit = ((long long)blockIdx.x * 256 + threadIdx.x) >> 5;
  if (unit >= a.total) return;
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const long long tile = unit / a.chunks;
  const int k0 = int(unit - tile * a.chunks) * (64 * kWarpBlocks<kGroup32>);
  const uint4* src = a.codes + (tile * a.k_blocks + k0 / 64) * 32 + lane;
#pragma unroll
  for (int b = 0; b < kWarpBlocks<kGroup32>; ++b) {
    if (k0 / 64 + b >= a.k_blocks) return;
    const uint4 u = __ldg(src + b * 32);
    const uint32_t words[4] = {u.x, u.y, u.z, u.w};
    // Two runs of 4 floats 16 apart, from the words of the lanes 4 g + t / 2 and 4 g + 2 + t / 2: four lanes' stores then fill
    // 64 bytes of a row (with 8 in a row, 16 of every 32: 36 us for 4096 x 8192 instead of 26).  8 bf16 fill their sectors.
    constexpr bool kTwoRuns = sizeof(T) == 4;
#pragma unroll
    for (int f = 0; f < 2; ++f) {
      const int i = int(tile) * 16 + g + 8 * f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        uint32_t word[2] = {words[2 * h + f], 0u};
        if (kTwoRuns) {
          const uint32_t mine = word[0];
#pragma unroll
          for (int j = 0; j < 2; ++j) word[j] = __shfl_sync(0xffffffffu, mine, (lane & 28) + 2 * j + (t >> 1)) >> (8 * (t & 1));
        }
        const int at = k0 + b * 64 + h * 32;
        if (i >= a.m || at >= a.k) continue;
        const long long s_at = (tile * a.n_groups + at / (32 * kGroup32)) * 16 + g + 8 * f;
        const float s = bf16_float(__ldg(a.scales + s_at)), z = 8388608.f + (a.zeros ? float(__ldg(a.zeros + s_at)) : 8.f);
        T* dst = w + (long long)i * a.pitch + at;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {                // 2^23 + code has the code in its mantissa
          const uint32_t bits = kTwoRuns ? word[e >> 2] >> shift_of(e & 3) : word[0] >> shift_of(e);
          v[e] = (__uint_as_float((bits & 15u) | 0x4B000000u) - z) * s;
        }
        if constexpr (kTwoRuns) {
#pragma unroll
          for (int j = 0; j < 2; ++j) store4<kVec>(dst + 16 * j + 4 * t, a.k - (at + 16 * j + 4 * t), v + 4 * j);
        } else {
          store8<kVec>(dst + 8 * t, a.k - (at + 8 * t), v);
        }
      }
    }
  }
}

// ------------------------------------------------------------------------------------------------ products of a few rows
// y[r][i] = sum_g s[i][g] sum_{k in g} (c[i][k] - z[i][g]) x[r][k].  A code minus its zero point is a whole number of at most 15,
// exact in bf16, and so is a bf16 x: the tensor cores' 16 x 8 x 16 products add up 32 inputs of a group
// without a rounding but the fp32 sum's, and the scale multiplies that sum in fp32.  fp32 rows go in as three bf16
// parts that add up to the value.  16 filters are the products' rows, 8 rows of x their columns: the tile layout holds for each lane
// the 16 bytes it needs, so a warp reads 512 bytes in a row, and nothing goes through shared memory but the sums at the end.
// (c - z): four bits at the bottom of a bf16 are the subnormal c 2^-133, at bits 4 to 7 (the lowest bit of the exponent among them)
// c 2^-129: one fused multiply-add makes (c - z) / 64 of either, exactly, and the result takes the 64 back.  9 instructions for
// eight weights, 5 of them on the integer pipe, which bounds the kernel where the codes come from the L2.
//
// A CTA's eight warps take every eighth block of 64 inputs of kTiles tiles of filters; where there are few tiles, the CTAs of a cluster
// share the inputs further and add their sums up through one another's shared memory, always in the same order.
constexpr int kLinearThreads = 256;
// More rows go to linear_w4_many_rows.  us here and there, groups of 128: 4096 x 8192, bf16: 16 rows 10.8 and 13.7, 32 rows 16.3 and 13.8;
// fp32: 16 rows 33.3 and 24.2, 64 rows 101 and 26 (groups of 32, 16 rows: 36.3 and 35.4).  487 x 4096, bf16: 16 rows 5.1 and 6.7, 32 rows 5.6
// and 6.8; fp32: 16 rows 13.7 and 10.1.  One number for all: fp32 rows from 9 on would be faster there, 32 bf16 rows of narrow layers here.
constexpr int kManyRows = 16;

__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
// The first `bytes` come from global memory, the rest of the 16 are zeros.
__device__ __forceinline__ void copy16_part(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory"); }

// Eight inputs of a row as bf16 pairs, 512 bytes between a lane's units.
template <typename T>
struct Operand;
template <>
struct Operand<__nv_bfloat16> {
  static constexpr int kParts = 1, kUnits = 1;
  static __device__ __forceinline__ void read(const unsigned char* at, uint32_t (&b)[kParts][4]) {
    const uint4 v = *reinterpret_cast<const uint4*>(at);
    b[0][0] = v.x; b[0][1] = v.y; b[0][2] = v.z; b[0][3] = v.w;
  }
};
template <>
struct Operand<float> {
  static constexpr int kParts = 3, kUnits = 2;
  static __device__ __forceinline__ void read(const unsigned char* at, uint32_t (&b)[kParts][4]) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const float4 v = *reinterpret_cast<const float4*>(at + u * 512);
      split_pair(v.x, v.y, b[0][2 * u], b[1][2 * u], b[2][2 * u]);
      split_pair(v.z, v.w, b[0][2 * u + 1], b[1][2 * u + 1], b[2][2 * u + 1]);
    }
  }
};

// A stage of a warp's ring: kDeep neighbouring blocks of 64 inputs: the codes [block][tile], the rows of x [block], then the
// groups' scales [tile][group] and zero points.
template <typename T, int kTiles, int kRows8, bool kFine>
struct Ring {
  static constexpr int kDeep = sizeof(T) == 4 && kRows8 == 2 ? 1 : sizeof(T) == 2 && kTiles <= 2 && kRows8 == 1 ? 4 : 2;
  static constexpr int kGroups = kFine ? 2 * kDeep : kDeep, kX = kRows8 * 2 * Operand<T>::kUnits;
  static constexpr uint32_t kXBlock = kX * 512, kXAt = kDeep * kTiles * 512, kGridAt = kXAt + kDeep * kXBlock;
  static constexpr uint32_t kZeroAt = kGridAt + kTiles * kGroups * 32;
  static constexpr uint32_t kStage = (kZeroAt + kTiles * kGroups * 16 + 127) / 128 * 128;
  static constexpr int kFit = int(104 * 1024 / 8 / kStage), kDepth = kFit >= 6 ? 6 : kFit >= 2 ? kFit : 2;
  static constexpr uint32_t kSums = 8 * kTiles * 16 * kRows8 * 8 * 4, kRings = 8 * kDepth * kStage, kBytes = kRings > kSums ? kRings : kSums;
};

// Sums of kNt <= kTiles tiles from `tile0` on over this warp's stages.
template <typename T, int kTiles, int kNt, int kRows8, bool kFine, bool kZeros>
__device__ __forceinline__ void linear_sums(const LinearArgs& a, unsigned char* ring, int tile0, long long row0, int first, int step, int lane,
                                            float (&acc)[kTiles][kRows8][4]) {
  typedef Ring<T, kTiles, kRows8, kFine> R;
  constexpr int kParts = Operand<T>::kParts, kUnits = Operand<T>::kUnits;
  const int g = lane >> 2, t = lane & 3;
  const int n = first < a.k_blocks ? (a.k_blocks - first + step - 1) / step : 0;   // this warp's stages
  const int stage_groups = kFine ? 2 * R::kDeep : (R::kDeep + a.group_shift) >> a.group_shift;      // groups of a stage

  // What this lane copies of a stage, as addresses that go on from stage to stage: its 16 bytes of every tile's codes, its eight
  // inputs of rows g, g + 8, .. and up to two of the 16-byte units of the scales (two a group) and zero points (one).
  const unsigned char* codes = reinterpret_cast<const unsigned char*>(a.codes) + ((long long)tile0 * a.k_blocks + first) * 512 + lane * 16;
  const long long tile_step = (long long)a.k_blocks * 512;
  const unsigned char* rows[kRows8];
#pragma unroll
  for (int r = 0; r < kRows8; ++r)
    rows[r] = row0 + r * 8 + g < a.rows
                  ? static_cast<const unsigned char*>(a.x) + ((row0 + r * 8 + g) * a.x_pitch + first * 64 + t * 8) * int(sizeof(T)) : nullptr;
  constexpr int kScaleUnits = kTiles * R::kGroups * 2, kGridUnits = kScaleUnits + (kZeros ? kTiles * R::kGroups : 0);
  constexpr int kMine = (kGridUnits + 31) / 32;
  const unsigned char* grid[kMine];                  // nullptr: nothing
  int grid_group[kMine];
#pragma unroll
  for (int c = 0; c < kMine; ++c) {
    const int u = lane + 32 * c;
    const bool z = u >= kScaleUnits;
    const int of_tile = z ? (u - kScaleUnits) % R::kGroups : u % (2 * R::kGroups) / 2;
    const int i = z ? (u - kScaleUnits) / R::kGroups : u / (2 * R::kGroups);
    grid_group[c] = (kFine ? first * 2 : first >> a.group_shift) + of_tile;
    const long long at = (long long)(tile0 + i) * a.n_groups + grid_group[c];
    grid[c] = u >= kGridUnits || i >= kNt || of_tile >= stage_groups ? nullptr
              : z ? a.zeros + at * 16 : reinterpret_cast<const unsigned char*>(a.scales) + at * 32 + (u & 1) * 16;
  }
  const int group_step = kFine ? 2 * step : step >> a.group_shift;
  const uint32_t ring_s = smem_u32(ring) + lane * 16;

  // rows that do not exist are zeros, once and for all
#pragma unroll
  for (int r = 0; r < kRows8; ++r)
    if (!rows[r])
      for (int s = 0; s < R::kDepth; ++s)
        for (int d = 0; d < R::kDeep; ++d)
#pragma unroll
          for (int u = 0; u < 2 * kUnits; ++u)
            *reinterpret_cast<uint4*>(ring + s * R::kStage + R::kXAt + d * R::kXBlock + (r * 2 * kUnits + u) * 512 + lane * 16) = make_uint4(0u, 0u, 0u, 0u);

  int f_kb = first;                                  // the next stage to be copied
  uint32_t f_at = ring_s;
  auto fetch = [&] {
    if (f_kb < a.k_blocks) {
      const bool whole = (f_kb + R::kDeep) * 64 <= a.k;
      if (whole) {
#pragma unroll
        for (int i = 0; i < kNt; ++i) {
          const unsigned char* p = codes + i * tile_step;
#pragma unroll
          for (int d = 0; d < R::kDeep; ++d) copy16(f_at + (d * kTiles + i) * 512, p + d * 512);
        }
#pragma unroll
        for (int r = 0; r < kRows8; ++r)
          if (rows[r]) {
#pragma unroll
            for (int d = 0; d < R::kDeep; ++d)
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int u = 0; u < kUnits; ++u)
                  copy16(f_at + R::kXAt + d * R::kXBlock + ((r * 2 + h) * kUnits + u) * 512, rows[r] + (d * 64 + h * 32 + u * 4) * int(sizeof(T)));
          }
#pragma unroll
        for (int c = 0; c < kMine; ++c)
          if (grid[c]) copy16(f_at + R::kGridAt + c * 512, grid[c]);
      } else {                                       // the last one, where it ends early: what lies behind the last input is not read
#pragma unroll 1
        for (int d = 0; d < R::kDeep && f_kb + d < a.k_blocks; ++d) {
#pragma unroll 1
          for (int i = 0; i < kNt; ++i) copy16(f_at + (d * kTiles + i) * 512, codes + i * tile_step + d * 512);
#pragma unroll
          for (int r = 0; r < kRows8; ++r)
            if (rows[r]) {
#pragma unroll
              for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int u = 0; u < kUnits; ++u) {
                  const int in = d * 64 + h * 32 + u * 4, left = (a.k - (f_kb * 64 + in + t * 8)) * int(sizeof(T));
                  copy16_part(f_at + R::kXAt + d * R::kXBlock + ((r * 2 + h) * kUnits + u) * 512, left > 0 ? rows[r] + in * int(sizeof(T)) : static_cast<const unsigned char*>(a.x),
                              max(0, min(16, left)));
                }
            }
        }
#pragma unroll
        for (int c = 0; c < kMine; ++c)
          if (grid[c])                               // zeros for groups that do not exist
            copy16_part(f_at + R::kGridAt + c * 512, grid_group[c] < a.n_groups ? grid[c] : static_cast<const unsigned char*>(a.x),
                        grid_group[c] < a.n_groups ? 16 : 0);
      }
      f_kb += step;
      codes += step * 512;
#pragma unroll
      for (int r = 0; r < kRows8; ++r)
        if (rows[r]) rows[r] += step * 64 * int(sizeof(T));
#pragma unroll
      for (int c = 0; c < kMine; ++c)
        if (grid[c]) {
          grid_group[c] += group_step;
          grid[c] += group_step * (lane + 32 * c >= kScaleUnits ? 16 : 32);
        }
      f_at = f_at + R::kStage == ring_s + R::kDepth * R::kStage ? ring_s : f_at + R::kStage;
    }
    copies_commit();
  };

  auto use = [&](const unsigned char* at, int d) {    // block d of the stage at `at`
    const unsigned char *mine = at + d * (kTiles * 512) + lane * 16, *x_at = at + R::kXAt + d * R::kXBlock + lane * 16;
    uint32_t xb[2][kRows8][kParts][4];
    constexpr bool kBoth = kParts == 1 && kRows8 <= 2;                         // both halves' rows in registers at a time
    if (kBoth) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int r = 0; r < kRows8; ++r) Operand<T>::read(x_at + (r * 2 + h) * kUnits * 512, xb[h][r]);
    }
    // one half of one tile: 32 inputs
    auto half = [&](int i, int h, const uint4& w, float (&sum)[kRows8][4]) {
      const int q = i * R::kGroups + (kFine ? 2 * d + h : d >> a.group_shift);
      uint32_t z0 = kMinusEighth, z1 = kMinusEighth, va[4], vb[4];
      if (kZeros) {
        z0 = minus_zero(at[R::kZeroAt + q * 16 + g]);
        z1 = minus_zero(at[R::kZeroAt + q * 16 + g + 8]);
      }
      spread_codes(h ? w.z : w.x, z0, va);
      spread_codes(h ? w.w : w.y, z1, vb);
#pragma unroll
      for (int r = 0; r < kRows8; ++r)
#pragma unroll
        for (int c = kParts - 1; c >= 0; --c) {                                // the smallest parts first
          const uint32_t (&x)[4] = xb[kBoth ? h : 0][r][c];
          mma_bf16(sum[r], va[0], vb[0], va[1], vb[1], x[0], x[1]);
          mma_bf16(sum[r], va[2], vb[2], va[3], vb[3], x[2], x[3]);
        }
    };
    auto scaled = [&](int i, int h, const float (&sum)[kRows8][4]) {
      const uint16_t* sc = reinterpret_cast<const uint16_t*>(at + R::kGridAt) + (i * R::kGroups + (kFine ? 2 * d + h : d >> a.group_shift)) * 16 + g;
      const float s0 = bf16_float(sc[0]), s1 = bf16_float(sc[8]);
#pragma unroll
      for (int r = 0; r < kRows8; ++r) {
        acc[i][r][0] = fmaf(s0, sum[r][0], acc[i][r][0]); acc[i][r][1] = fmaf(s0, sum[r][1], acc[i][r][1]);
        acc[i][r][2] = fmaf(s1, sum[r][2], acc[i][r][2]); acc[i][r][3] = fmaf(s1, sum[r][3], acc[i][r][3]);
      }
    };
    if (kBoth) {
#pragma unroll
      for (int i = 0; i < kNt; ++i) {
        const uint4 w = *reinterpret_cast<const uint4*>(mine + i * 512);
        float sum[kRows8][4] = {};
        half(i, 0, w, sum);
        if (kFine) {
          scaled(i, 0, sum);
#pragma unroll
          for (int r = 0; r < kRows8; ++r) sum[r][0] = sum[r][1] = sum[r][2] = sum[r][3] = 0.f;
        }
        half(i, 1, w, sum);
        scaled(i, 1, sum);
      }
    } else {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int r = 0; r < kRows8; ++r) Operand<T>::read(x_at + (r * 2 + h) * kUnits * 512, xb[0][r]);
#pragma unroll
        for (int i = 0; i < kNt; ++i) {
          const uint4 w = *reinterpret_cast<const uint4*>(mine + i * 512);
          float sum[kRows8][4] = {};
          half(i, h, w, sum);
          scaled(i, h, sum);
        }
      }
    }
  };

#pragma unroll 1
  for (int s = 0; s < R::kDepth - 1; ++s) fetch();
  const unsigned char* at = ring;
  int kb = first;
#pragma unroll 1
  for (int s = 0; s < n; ++s, kb += step) {
    copies_wait<R::kDepth - 2>();
    __syncwarp();                                    // every lane's copies of this stage are there, and nobody reads the last one any more
    fetch();
#pragma unroll
    for (int d = 0; d < R::kDeep; ++d)
      if (kb + d < a.k_blocks) use(at, d);
    at = at + R::kStage == ring + R::kDepth * R::kStage ? ring : at + R::kStage;
  }
  copies_wait<0>();
}

template <typename T, int kTiles, int kRows8, bool kFine, bool kZeros>        // kFine: groups of 32, two to a block
__global__ void __launch_bounds__(kLinearThreads, 2)
linear_w4_kernel(const LinearArgs a) {
  typedef Ring<T, kTiles, kRows8, kFine> R;
  constexpr int kCols = kRows8 * 8, kOut = kTiles * 16 * kCols;
  extern __shared__ __align__(128) unsigned char smem_raw[];
  float* part = reinterpret_cast<float*>(smem_raw);                           // [8][kOut], where the rings were
  pdl_entry();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t ranks = cluster_size(), rank = cluster_ctarank();
  // This CTA's tiles: as many as the others', or one less.  CTAs n and n + n_sms run on one SM, as a rule, and share the tiles
  // of n_sms th parts.
  const int cta = int(blockIdx.x / ranks), n_ctas = int(gridDim.x / ranks);
  const int tile0 = int((long long)cta * a.n_tiles / n_ctas), nt = int((long long)(cta + 1) * a.n_tiles / n_ctas) - tile0;
  const long long row0 = (long long)blockIdx.y * kCols;
  const int step = 8 * R::kDeep * int(ranks), first = (int(rank) * 8 + warp) * R::kDeep;
  unsigned char* ring = smem_raw + warp * (R::kDepth * R::kStage);
  float acc[kTiles][kRows8][4] = {};
  if (nt == kTiles) linear_sums<T, kTiles, kTiles, kRows8, kFine, kZeros>(a, ring, tile0, row0, first, step, lane, acc);
  else if constexpr (kTiles > 1) linear_sums<T, kTiles, kTiles - 1, kRows8, kFine, kZeros>(a, ring, tile0, row0, first, step, lane, acc);
  __syncthreads();

  // the warps' sums, [filter][row of x]
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int r = 0; r < kRows8; ++r) {
      float* at = part + warp * kOut + (i * 16 + g) * kCols + r * 8 + 2 * t;
      *reinterpret_cast<float2*>(at) = make_float2(acc[i][r][0], acc[i][r][1]);
      *reinterpret_cast<float2*>(at + 8 * kCols) = make_float2(acc[i][r][2], acc[i][r][3]);
    }
  __syncthreads();
  if (ranks > 1) {
    for (int o = threadIdx.x; o < kOut; o += kLinearThreads) {
      float s = part[o];
#pragma unroll
      for (int w = 1; w < 8; ++w) s += part[w * kOut + o];
      part[o] = s;
    }
    cluster_sync_all();
  }
  T* y = static_cast<T*>(a.y);
  // filters fastest, so that neighbouring threads write neighbouring values of y
  for (int v = threadIdx.x + int(rank) * kLinearThreads; v < kOut; v += kLinearThreads * int(ranks)) {
    const int f = v % (kTiles * 16), r = v / (kTiles * 16), o = f * kCols + r;
    float s;
    if (ranks > 1) {
      s = 0.f;
      for (uint32_t p = 0; p < ranks; ++p) s += ld_cluster_f32(mapa_shared(smem_u32(part + o), p));
    } else {
      s = part[o];
#pragma unroll
      for (int w = 1; w < 8; ++w) s += part[w * kOut + o];
    }
    const int i = tile0 * 16 + f;
    if (f < nt * 16 && i < a.m && row0 + r < a.rows) {
      s *= 64.f;
      if (a.bias) s += __ldg(a.bias + i);
      store_value(y + (row0 + r) * a.y_pitch + i, a.relu ? relu_of(s) : s);
    }
  }
  if (ranks > 1) cluster_sync_all();                 // nobody leaves while its sums are still being read
}

bool valid_extents(int64_t m, int64_t k) { return m > 0 && k > 0; }
// Tiles of codes are counted, and filters (up to whole tiles) and inputs addressed, in 32 bits.
bool small_enough(int64_t m, int64_t k) { return m <= (int64_t(1) << 31) - 64 && k <= (1 << 30) && ceil_div64(m, 16) * ceil_div64(k, 64) < (int64_t(1) << 31); }
bool valid_group(int group) { return group == 32 || group == 64 || group == 128; }

rt3d_status check_w4(const rt3d_w4* q) {
  if (!q || !q->codes || !q->scales || !valid_extents(q->m, q->k) || !valid_group(q->group)) return RT3D_ERR_INVALID_ARG;
  const uintptr_t bits = reinterpret_cast<uintptr_t>(q->codes) | reinterpret_cast<uintptr_t>(q->scales) | reinterpret_cast<uintptr_t>(q->zeros);
  if (bits & 15) return RT3D_ERR_INVALID_ARG;
  if (!small_enough(q->m, q->k)) return RT3D_ERR_UNSUPPORTED;
  return RT3D_OK;
}
// Arguments of the calls that read or write a plain matrix.
rt3d_status check_matrix(const void* w, int dtype, int64_t pitch, const rt3d_w4* q) {
  const rt3d_status s = check_w4(q);
  if (s != RT3D_OK) return s;
  if (!w || (dtype != RT3D_F32 && dtype != RT3D_BF16) || pitch < q->k) return RT3D_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(w) % (dtype == RT3D_BF16 ? 2 : 4)) return RT3D_ERR_INVALID_ARG;
  return RT3D_OK;
}
rt3d_status launched(cudaError_t e) {
  if (e != cudaSuccess) return RT3D_ERR_CUDA;
  count_launches(1);
  return RT3D_OK;
}
// Rows of a product, -1 for 2^31 and more.
int64_t rows_of(const rt3d_tensor* t) {
  int64_t n = 1;
  for (const int32_t e : {t->n, t->t, t->h, t->w})
    if ((n *= e) >= (int64_t(1) << 31)) return -1;
  return n;
}
template <typename T, bool kQuantize, int kGroup32>
rt3d_status launch_between(T* w, int64_t pitch, const rt3d_w4* q, cudaStream_t st) {
  GridArgs a;
  a.codes = reinterpret_cast<uint4*>(q->codes);
  a.scales = q->scales; a.zeros = q->zeros; a.pitch = pitch;
  a.m = q->m; a.k = q->k; a.n_groups = ceil_div(q->k, q->group); a.k_blocks = ceil_div(q->k, 64);
  a.chunks = ceil_div(q->k, 64 * kWarpBlocks<kGroup32>); a.total = a.chunks * ceil_div(q->m, 16);
  const bool vec = (reinterpret_cast<uintptr_t>(w) | uintptr_t(pitch) * sizeof(T)) % 16 == 0;
  LaunchSetup ls(dim3(unsigned((a.total + 7) / 8)), dim3(256), 0, st);                  // 8 warps a block: total < 2^31
  if constexpr (kQuantize)
    return launched(vec ? cudaLaunchKernelEx(&ls.cfg, w4_quantize_kernel<T, kGroup32, true>, (const T*)w, a)
                        : cudaLaunchKernelEx(&ls.cfg, w4_quantize_kernel<T, kGroup32, false>, (const T*)w, a));
  else
    return launched(vec ? cudaLaunchKernelEx(&ls.cfg, w4_unpack_kernel<T, kGroup32, true>, w, a)
                        : cudaLaunchKernelEx(&ls.cfg, w4_unpack_kernel<T, kGroup32, false>, w, a));
}
template <typename T, bool kQuantize>
rt3d_status between(T* w, int64_t pitch, const rt3d_w4* q, void* stream) {
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return q->group == 32 ? launch_between<T, kQuantize, 1>(w, pitch, q, st) : q->group == 64 ? launch_between<T, kQuantize, 2>(w, pitch, q, st)
                                                                                            : launch_between<T, kQuantize, 4>(w, pitch, q, st);
}

template <typename T, int kTiles, int kRows8>
rt3d_status launch_linear(const LinearArgs& a, bool fine, int ctas, int ranks, cudaStream_t st) {
  const dim3 grid(unsigned(ctas * ranks), unsigned(ceil_div(a.rows, kRows8 * 8)));
  const uint32_t smem = fine ? Ring<T, kTiles, kRows8, true>::kBytes : Ring<T, kTiles, kRows8, false>::kBytes;
  LaunchSetup ls(grid, dim3(kLinearThreads), smem, st, unsigned(ranks));
  void (*const kernels[2][2])(LinearArgs) = {{linear_w4_kernel<T, kTiles, kRows8, false, false>, linear_w4_kernel<T, kTiles, kRows8, false, true>},
                                             {linear_w4_kernel<T, kTiles, kRows8, true, false>, linear_w4_kernel<T, kTiles, kRows8, true, true>}};
  const auto kernel = kernels[fine][a.zeros != nullptr];
  static std::atomic<bool> attr_done[kMaxDevices][2][2];        // the attribute is per device
  const int dev = current_device_index();
  if (dev < 0) return RT3D_ERR_CUDA;
  std::atomic<bool>& done = attr_done[dev][fine][a.zeros != nullptr];
  if (!done.load()) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem)) != cudaSuccess) return RT3D_ERR_CUDA;
    done.store(true);
  }
  return launched(cudaLaunchKernelEx(&ls.cfg, kernel, a));
}
template <typename T>
rt3d_status linear(const rt3d_tensor* x, const rt3d_w4* q, const float* bias, int relu, rt3d_tensor* y, long long rows, const DeviceInfo& dev, cudaStream_t st) {
  const int sms = dev.sm_count;
  LinearArgs a;
  a.codes = reinterpret_cast<const uint4*>(q->codes);
  a.scales = q->scales; a.zeros = q->zeros; a.bias = bias; a.x = x->data; a.y = y->data;
  a.x_pitch = x->c_stride; a.y_pitch = y->c_stride;
  a.m = q->m; a.k = q->k; a.group_shift = q->group == 128 ? 1 : 0; a.fine = q->group == 32 ? 1 : 0; a.n_groups = ceil_div(q->k, q->group);
  a.k_blocks = ceil_div(q->k, 64); a.n_tiles = ceil_div(q->m, 16); a.relu = relu ? 1 : 0; a.rows = int(rows);
  if (rows > kMostRows) {                                     // the grid's second extent: one launch after another
    for (long long r = 0; r < rows; r += kMostRows) {
      rt3d_tensor xs = *x, ys = *y;
      xs.data = static_cast<T*>(x->data) + r * x->c_stride;
      ys.data = static_cast<T*>(y->data) + r * y->c_stride;
      const rt3d_status s = linear<T>(&xs, q, bias, relu, &ys, rows - r < kMostRows ? rows - r : kMostRows, dev, st);
      if (s != RT3D_OK) return s;
    }
    return RT3D_OK;
  }
  if (rows > kManyRows) return linear_w4_many_rows(a, x->dtype, dev, st);
  const int rows8 = rows <= 8 ? 1 : 2;
  // tiles of a CTA at most: sixteen fp32 rows take three times the registers of bf16 ones
  const int most = rows8 == 2 && sizeof(T) == 4 ? 2 : 4;
  // One CTA an SM for up to two tiles each (4096 x 8192, one row: 7.2 us as 256 CTAs and as 148; 16 rows: 11.9 and 11.0), two for
  // more (16384 x 16384, 4 rows: 37.4 us as 342 CTAs of up to 3 tiles, 30.3 as 296 of up to 4).  With fewer tiles than that, the CTAs
  // of a cluster share the inputs while every warp keeps eight blocks (16384 inputs of 1000 filters, one row: 7.9 us alone, 5.9
  // shared by four; 4096 inputs of 487: 4.0 alone, 4.2 by two).
  const int ctas = a.n_tiles <= sms ? a.n_tiles : a.n_tiles <= 2 * sms ? sms : 2 * sms * ceil_div(a.n_tiles, most * 2 * sms);
  int ranks = 1;
  while (ranks < 8 && ctas < sms && ctas * ranks <= sms && a.k_blocks >= 128 * ranks) ranks *= 2;
  const int tiles = ceil_div(a.n_tiles, ctas);
  const bool fine = q->group == 32;
  if (rows8 == 1) {
    if (tiles == 1) return launch_linear<T, 1, 1>(a, fine, ctas, ranks, st);
    if (tiles == 2) return launch_linear<T, 2, 1>(a, fine, ctas, ranks, st);
    if (tiles == 3) return launch_linear<T, 3, 1>(a, fine, ctas, ranks, st);
    return launch_linear<T, 4, 1>(a, fine, ctas, ranks, st);
  }
  if (tiles == 1) return launch_linear<T, 1, 2>(a, fine, ctas, ranks, st);
  if constexpr (sizeof(T) == 2) {
    if (tiles == 3) return launch_linear<T, 3, 2>(a, fine, ctas, ranks, st);
    if (tiles == 4) return launch_linear<T, 4, 2>(a, fine, ctas, ranks, st);
  }
  return launch_linear<T, 2, 2>(a, fine, ctas, ranks, st);
}

}  // namespace
}  // namespace rt3d

using namespace rt3d;

extern "C" {

int64_t rt3d_w4_codes_bytes(int m, int k) {
  if (!valid_extents(m, k) || !small_enough(m, k)) return -1;
  return ceil_div64(m, 16) * ceil_div64(k, 64) * 512;
}

int64_t rt3d_w4_scale_count(int m, int k, int group) {
  if (rt3d_w4_codes_bytes(m, k) < 0 || !valid_group(group)) return -1;
  return ceil_div64(m, 16) * 16 * ceil_div64(k, group);
}

rt3d_status rt3d_w4_quantize(const void* w, int dtype, int64_t pitch, const rt3d_w4* q, void* stream) {
  const rt3d_status s = check_matrix(w, dtype, pitch, q);
  if (s != RT3D_OK) return s;
  if (plan_only()) return RT3D_OK;
  return dtype == RT3D_BF16 ? between<__nv_bfloat16, true>(static_cast<__nv_bfloat16*>(const_cast<void*>(w)), pitch, q, stream)
                            : between<float, true>(static_cast<float*>(const_cast<void*>(w)), pitch, q, stream);
}

rt3d_status rt3d_w4_unpack(const rt3d_w4* q, int dtype, void* w, int64_t pitch, void* stream) {
  const rt3d_status s = check_matrix(w, dtype, pitch, q);
  if (s != RT3D_OK) return s;
  if (plan_only()) return RT3D_OK;
  return dtype == RT3D_BF16 ? between<__nv_bfloat16, false>(static_cast<__nv_bfloat16*>(w), pitch, q, stream)
                            : between<float, false>(static_cast<float*>(w), pitch, q, stream);
}

rt3d_status rt3d_linear_w4(const rt3d_tensor* x, const rt3d_w4* q, const float* bias, int relu, rt3d_tensor* y, void* stream) {
  rt3d_status s;
  if ((s = check_device_tensor(x)) != RT3D_OK || (s = check_device_tensor(y)) != RT3D_OK || (s = check_w4(q)) != RT3D_OK) return s;
  if (x->n != y->n || x->t != y->t || x->h != y->h || x->w != y->w || x->dtype != y->dtype || x->c != q->k || y->c != q->m) return RT3D_ERR_SHAPE;
  const int64_t rows = rows_of(x);
  if (rows < 0) return RT3D_ERR_UNSUPPORTED;
  if (tensors_overlap(x, y)) return RT3D_ERR_INVALID_ARG;
  if (plan_only()) return RT3D_OK;
  DeviceInfo dev;
  if ((s = current_device_info(&dev)) != RT3D_OK) return s;
  if (dev.cc_major != 10) return RT3D_ERR_UNSUPPORTED;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return x->dtype == RT3D_BF16 ? linear<__nv_bfloat16>(x, q, bias, relu, y, rows, dev, st)
                               : linear<float>(x, q, bias, relu, y, rows, dev, st);
}

}  // extern "C"
