// What the kernels of products with 4-bit weights share.  Included by .cu files only, after umma_common.cuh.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "rt3d.h"
#include "rt3d_internal.h"

namespace rt3d {

struct LinearArgs {
  const uint4* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  const float* bias;
  const void* x;
  void* y;
  long long x_pitch, y_pitch;
  int m, k, group_shift, fine, n_groups, k_blocks, n_tiles, relu;
  int rows;
};

// Many rows (w4_umma.cu), at most kMostRows: tiles of 64 rows are the grid's second extent.
constexpr int kMostRows = 1 << 19;
static_assert(kMostRows / 64 <= 65535, "tiles of 64 rows");
rt3d_status linear_w4_many_rows(const LinearArgs& a, int dtype, const DeviceInfo& dev, cudaStream_t st);

namespace {

__device__ __forceinline__ float bf16_float(uint16_t b) { return __uint_as_float(uint32_t(b) << 16); }
// max(v, 0) that lets a NaN through.
__device__ __forceinline__ float relu_of(float v) { return v < 0.f ? 0.f : v; }
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

__device__ __forceinline__ uint32_t fma_bf16x2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
constexpr uint32_t kTwo127 = 0x7f007f00u, kTwo123 = 0x7d007d00u;               // bf16 2^127 and 2^123, twice
constexpr uint32_t kMinusEighth = 0xbe00be00u;                                 // -8 / 64, twice
// -z / 64, twice: 128 + z has z in its mantissa, and -(128 + z) / 64 + 2.
__device__ __forceinline__ uint32_t minus_zero(uint32_t z) { return fma_bf16x2(z * 0x00010001u + 0x43004300u, 0xbc80bc80u, 0x40004000u); }
// Eight codes of a word as four pairs of (code - zero) / 64, inputs (2 p, 2 p + 1).
__device__ __forceinline__ void spread_codes(uint32_t w, uint32_t minus, uint32_t (&v)[4]) {
  const uint32_t u = w >> 8;
  v[0] = fma_bf16x2(w & 0x000F000Fu, kTwo127, minus);
  v[1] = fma_bf16x2(w & 0x00F000F0u, kTwo123, minus);
  v[2] = fma_bf16x2(u & 0x000F000Fu, kTwo127, minus);
  v[3] = fma_bf16x2(u & 0x00F000F0u, kTwo123, minus);
}
// Three bf16 parts of two values, packed: the upper 8 bits of the mantissa, the next 8 and the last 8.  Each part is the rest's leading bits,
// so the three add up to the value and none is larger than it.  An infinity has no rest; a NaN's is a NaN.
__device__ __forceinline__ void split_pair(float x, float y, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
  const float v[2] = {x, y};
  uint32_t bits[3][2];
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const uint32_t h = __float_as_uint(v[e]) & 0xffff0000u;
    const float r = fabsf(v[e]) == __int_as_float(0x7f800000) ? 0.f : v[e] - __uint_as_float(h);
    const uint32_t m = __float_as_uint(r) & 0xffff0000u;
    bits[0][e] = h; bits[1][e] = m; bits[2][e] = __float_as_uint(r - __uint_as_float(m));
  }
  hi = __byte_perm(bits[0][0], bits[0][1], 0x7632);
  mid = __byte_perm(bits[1][0], bits[1][1], 0x7632);
  lo = __byte_perm(bits[2][0], bits[2][1], 0x7632);
}

__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

}  // namespace
}  // namespace rt3d
