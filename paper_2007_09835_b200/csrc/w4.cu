// 4-bit weights with group scales: quantisation, its inverse and the products with a few rows of activations.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "pdl.cuh"
#include "rt3d.h"
#include "rt3d_internal.h"
#include "umma_common.cuh"

namespace rt3d {
namespace {

__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}
// max(v, 0) that lets a NaN through.
__device__ __forceinline__ float relu_of(float v) { return v < 0.f ? 0.f : v; }

__device__ __forceinline__ float value_of(const float* p) { return *p; }
__device__ __forceinline__ float value_of(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ float bf16_float(uint16_t b) { return __uint_as_float(uint32_t(b) << 16); }

// Words of the code layout: filter i (of all), input block of 8 kw -> word index; shift of input e inside the word.
__device__ __forceinline__ long long word_of(int i, int kw, int k_blocks) {
  const int r = i & 15, b = kw >> 3, t = kw & 3, half = (kw >> 2) & 1;
  return ((long long)(i >> 4) * k_blocks + b) * 128 + ((r & 7) * 4 + t) * 4 + half * 2 + (r >> 3);
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
__device__ __forceinline__ uint32_t code_of(float v, const Grid& q) {
  if (!(q.scale > 0.f)) return 8u;
  return uint32_t(fminf(fmaxf(rintf(__fdiv_rn(v, q.scale)) + q.zero, 0.f), 15.f));
}

// One thread for a group of a filter; threads of filters that do not exist write the padding of the last tile.
template <typename T>
__global__ void w4_quantize_kernel(const T* __restrict__ w, long long pitch, int m, int k, int group, int n_groups, int k_blocks,
                                   uint32_t* __restrict__ codes, uint16_t* __restrict__ scales, uint8_t* __restrict__ zeros,
                                   long long total) {
  pdl_entry();
  const long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (idx >= total) return;
  const int g = int(idx % n_groups), i = int(idx / n_groups);
  const int k0 = g * group, n = min(group, k - k0);
  const T* src = w + (long long)i * pitch + k0;
  float low = 0.f, high = 0.f;
  bool bad = false;
  if (i < m)
    for (int j = 0; j < n; ++j) {
      const float v = value_of(src + j);
      low = fminf(low, v); high = fmaxf(high, v);
      bad |= !(fabsf(v) < __int_as_float(0x7f800000));
    }
  const Grid q = grid_of(low, high, bad, zeros != nullptr);
  const long long at = ((long long)(i >> 4) * n_groups + g) * 16 + (i & 15);
  scales[at] = q.bits;
  if (zeros) zeros[at] = uint8_t(q.zero);
  const int last = g == n_groups - 1 ? k_blocks * 8 : (k0 + group) / 8;
  for (int kw = k0 / 8; kw < last; ++kw) {
    uint32_t word = 0;
    for (int e = 0; e < 8; ++e) {
      const int j = kw * 8 + e - k0;
      word |= (i < m && j < n ? code_of(value_of(src + j), q) : uint32_t(q.zero)) << shift_of(e);
    }
    codes[word_of(i, kw, k_blocks)] = word;
  }
}

template <typename T>
__global__ void w4_unpack_kernel(const uint32_t* __restrict__ codes, const uint16_t* __restrict__ scales,
                                 const uint8_t* __restrict__ zeros, int m, int k, int group, int n_groups, int k_blocks, int words,
                                 T* __restrict__ w, long long pitch, long long total) {
  pdl_entry();
  const long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  if (idx >= total) return;
  const int kw = int(idx % words), i = int(idx / words);
  const long long at = ((long long)(i >> 4) * n_groups + kw * 8 / group) * 16 + (i & 15);
  const float s = bf16_float(scales[at]), z = zeros ? float(zeros[at]) : 8.f;
  const uint32_t word = codes[word_of(i, kw, k_blocks)];
  for (int e = 0; e < 8 && kw * 8 + e < k; ++e)
    store_value(w + (long long)i * pitch + kw * 8 + e, (float((word >> shift_of(e)) & 15u) - z) * s);
}

// ------------------------------------------------------------------------------------------------ products of a few rows
// y[r][i] = sum_g s[i][g] sum_{k in g} (c[i][k] - z[i][g]) x[r][k].  A code minus its zero point is a whole number of at most 15,
// exact in bf16, and so is a bf16 x: the tensor cores' 16 x 8 x 16 products add up 32 inputs of a group
// without a rounding but the fp32 sum's, and the scale multiplies that sum in fp32.  fp32 rows go in as three bf16
// parts that add up to the value.  16 filters are the products' rows, 8 rows of x their columns: the tile layout holds for each lane
// the 16 bytes it needs, so a warp reads 512 bytes in a row, and nothing goes through shared memory but the sums at the end.
// (c - z): the four bits go into the mantissa of 128 (bf16 has 7 bits), from which 128 + z is taken, exactly: 11 instructions for
// eight weights.
//
// A CTA's eight warps take every eighth block of 64 inputs of kTiles tiles of filters; where there are few tiles, the CTAs of a cluster
// share the inputs further and add their sums up through one another's shared memory, always in the same order.
constexpr int kLinearThreads = 256;
constexpr uint32_t kBias128 = 0x43004300u;                  // bf16 128, twice

__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
  const __nv_bfloat162 d = __hsub2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
  return *reinterpret_cast<const uint32_t*>(&d);
}
// Eight codes of a word as four pairs of whole numbers, inputs (2 p, 2 p + 1).
__device__ __forceinline__ void spread_codes(uint32_t w, uint32_t zero, uint32_t (&v)[4]) {
#pragma unroll
  for (int p = 0; p < 4; ++p) v[p] = sub_bf16x2(((w >> (4 * p)) & 0x000F000Fu) | kBias128, zero);
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Eight inputs of a row from k0 on as they lie in memory; zeros where there are none.
template <typename T>
struct Chunk;
template <>
struct Chunk<__nv_bfloat16> {
  static constexpr int kParts = 1;
  uint4 v;
  __device__ __forceinline__ void load(const __nv_bfloat16* row, int k0, int k) {
    v = make_uint4(0u, 0u, 0u, 0u);
    if (!row || k0 >= k) return;
    if (k0 + 8 <= k) { v = __ldg(reinterpret_cast<const uint4*>(row + k0)); return; }
    uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k0 + e < k) w[e >> 1] |= uint32_t(__bfloat16_as_ushort(row[k0 + e])) << (16 * (e & 1));
    v = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void parts(uint32_t (&b)[kParts][4]) const { b[0][0] = v.x; b[0][1] = v.y; b[0][2] = v.z; b[0][3] = v.w; }
};
template <>
struct Chunk<float> {
  static constexpr int kParts = 3;
  float f[8];
  __device__ __forceinline__ void load(const float* row, int k0, int k) {
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = 0.f;
    if (!row || k0 >= k) return;
    if (k0 + 8 <= k) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(row + k0)), b = __ldg(reinterpret_cast<const float4*>(row + k0 + 4));
      f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
      return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (k0 + e < k) f[e] = row[k0 + e];
  }
  // The upper 8 bits of the mantissa, the next 8 and the last 8: each part is the rest's leading bits, so the three add up to the
  // value and none is larger than it.  An infinity has no rest; a NaN's is a NaN.
  __device__ __forceinline__ void parts(uint32_t (&b)[kParts][4]) const {
#pragma unroll
    for (int p = 0; p < 4; ++p) {
      uint32_t bits[3][2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float x = f[2 * p + e];
        const uint32_t h = __float_as_uint(x) & 0xffff0000u;
        const float r = fabsf(x) == __int_as_float(0x7f800000) ? 0.f : x - __uint_as_float(h);
        const uint32_t m = __float_as_uint(r) & 0xffff0000u;
        bits[0][e] = h; bits[1][e] = m; bits[2][e] = __float_as_uint(r - __uint_as_float(m));
      }
#pragma unroll
      for (int q = 0; q < 3; ++q) b[q][p] = __byte_perm(bits[q][0], bits[q][1], 0x7632);
    }
  }
};

struct LinearArgs {
  const uint4* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  const float* bias;
  const void* x;
  void* y;
  long long x_pitch, y_pitch;
  int m, k, group_shift, n_groups, k_blocks, n_tiles, relu;
  int rows;
};

template <typename T, int kTiles, int kRows8, bool kFine, bool kZeros>        // kFine: groups of 32, two to a block
__global__ void __launch_bounds__(kLinearThreads, 2)
linear_w4_kernel(const LinearArgs a) {
  constexpr int kCols = kRows8 * 8, kOut = kTiles * 16 * kCols, kParts = Chunk<T>::kParts;
  __shared__ __align__(16) float part[8][kOut];
  pdl_entry();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const uint32_t ranks = cluster_size(), rank = cluster_ctarank();
  const int tile0 = int(blockIdx.x / ranks) * kTiles;
  const long long row0 = (long long)blockIdx.y * kCols;
  const T* rows[kRows8];
#pragma unroll
  for (int r = 0; r < kRows8; ++r)
    rows[r] = row0 + r * 8 + g < a.rows ? static_cast<const T*>(a.x) + (row0 + r * 8 + g) * a.x_pitch : nullptr;

  // One block of 64 inputs: the codes of kTiles tiles, and their scales (and zero points), of which lane 4 g + t loads filter
  // g + 8 (t & 1) of the block's half t / 2.  Both, and bf16 rows of up to 16, are asked for a block ahead.
  constexpr bool kAhead = sizeof(T) == 2 && kRows8 <= 2;
  struct Block {
    uint4 codes[kTiles];
    uint32_t scale[kTiles], zero[kTiles];
    Chunk<T> x[kAhead ? kRows8 : 1][2];
  };
  auto fetch = [&](Block& b, int kb) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
      const int tile = min(tile0 + i, a.n_tiles - 1);                          // a tile too many: computed and dropped
      b.codes[i] = __ldg(a.codes + ((long long)tile * a.k_blocks + kb) * 32 + lane);
      const int grp = min(kFine ? kb * 2 + (t >> 1) : kb >> a.group_shift, a.n_groups - 1);
      const long long at = ((long long)tile * a.n_groups + grp) * 16 + g + 8 * (t & 1);
      b.scale[i] = __ldg(a.scales + at);
      if (kZeros) b.zero[i] = __ldg(a.zeros + at);
    }
    if constexpr (kAhead) {
#pragma unroll
      for (int r = 0; r < kRows8; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) b.x[r][h].load(rows[r], kb * 64 + h * 32 + t * 8, a.k);
    }
  };

  float acc[kTiles][kRows8][4] = {};
  auto use = [&](const Block& b, int kb) {
    uint32_t grid[kTiles];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) grid[i] = kZeros ? b.scale[i] << 16 | b.zero[i] : b.scale[i] << 16;
#pragma unroll
    for (int h = 0; h < 2; ++h) {                                              // 32 inputs, one group's
      uint32_t xb[kRows8][kParts][4];
#pragma unroll
      for (int r = 0; r < kRows8; ++r) {
        if constexpr (kAhead) {
          b.x[r][h].parts(xb[r]);
        } else {
          Chunk<T> c;
          c.load(rows[r], kb * 64 + h * 32 + t * 8, a.k);
          c.parts(xb[r]);
        }
      }
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        uint32_t q[2], va[4], vb[4];                                           // of the filters g and g + 8
#pragma unroll
        for (int f = 0; f < 2; ++f) q[f] = __shfl_sync(0xffffffffu, grid[i], (lane & 28) + (kFine ? 2 * h : 0) + f);
        const uint32_t words[2] = {h ? b.codes[i].z : b.codes[i].x, h ? b.codes[i].w : b.codes[i].y};
        spread_codes(words[0], kZeros ? kBias128 + (q[0] & 0xffu) * 0x00010001u : 0x43084308u, va);
        spread_codes(words[1], kZeros ? kBias128 + (q[1] & 0xffu) * 0x00010001u : 0x43084308u, vb);
        const float s0 = __uint_as_float(q[0] & 0xffff0000u), s1 = __uint_as_float(q[1] & 0xffff0000u);
#pragma unroll
        for (int r = 0; r < kRows8; ++r) {
          float sum[4] = {};
#pragma unroll
          for (int c = kParts - 1; c >= 0; --c) {                              // the smallest parts first
            mma_bf16(sum, va[0], vb[0], va[1], vb[1], xb[r][c][0], xb[r][c][1]);
            mma_bf16(sum, va[2], vb[2], va[3], vb[3], xb[r][c][2], xb[r][c][3]);
          }
          acc[i][r][0] = fmaf(s0, sum[0], acc[i][r][0]); acc[i][r][1] = fmaf(s0, sum[1], acc[i][r][1]);
          acc[i][r][2] = fmaf(s1, sum[2], acc[i][r][2]); acc[i][r][3] = fmaf(s1, sum[3], acc[i][r][3]);
        }
      }
    }
  };

  const int step = 8 * int(ranks);
  int kb = int(rank) * 8 + warp;
  if (kb < a.k_blocks) {
    Block now, next;
    fetch(now, kb);
    for (; kb + step < a.k_blocks; kb += step) {
      fetch(next, kb + step);
      use(now, kb);
      now = next;
    }
    use(now, kb);
  }

  // the warps' sums, [filter][row of x]
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int r = 0; r < kRows8; ++r) {
      float* at = part[warp] + (i * 16 + g) * kCols + r * 8 + 2 * t;
      *reinterpret_cast<float2*>(at) = make_float2(acc[i][r][0], acc[i][r][1]);
      *reinterpret_cast<float2*>(at + 8 * kCols) = make_float2(acc[i][r][2], acc[i][r][3]);
    }
  __syncthreads();
  if (ranks > 1) {
    for (int o = threadIdx.x; o < kOut; o += kLinearThreads) {
      float s = part[0][o];
#pragma unroll
      for (int w = 1; w < 8; ++w) s += part[w][o];
      part[0][o] = s;
    }
    cluster_sync_all();
  }
  T* y = static_cast<T*>(a.y);
  // filters fastest, so that neighbouring threads write neighbouring values of y
  for (int n = threadIdx.x + int(rank) * kLinearThreads; n < kOut; n += kLinearThreads * int(ranks)) {
    const int f = n % (kTiles * 16), r = n / (kTiles * 16), o = f * kCols + r;
    float s;
    if (ranks > 1) {
      s = 0.f;
      for (uint32_t p = 0; p < ranks; ++p) s += ld_cluster_f32(mapa_shared(smem_u32(&part[0][o]), p));
    } else {
      s = part[0][o];
#pragma unroll
      for (int w = 1; w < 8; ++w) s += part[w][o];
    }
    const int i = tile0 * 16 + f;
    if (i < a.m && row0 + r < a.rows) {
      if (a.bias) s += __ldg(a.bias + i);
      store_value(y + (row0 + r) * a.y_pitch + i, a.relu ? relu_of(s) : s);
    }
  }
  if (ranks > 1) cluster_sync_all();                 // nobody leaves while its sums are still being read
}

bool valid_extents(int64_t m, int64_t k) { return m > 0 && k > 0; }
bool valid_group(int group) { return group == 32 || group == 64 || group == 128; }

rt3d_status check_w4(const rt3d_w4* q) {
  if (!q || !q->codes || !q->scales || !valid_extents(q->m, q->k) || !valid_group(q->group)) return RT3D_ERR_INVALID_ARG;
  const uintptr_t bits = reinterpret_cast<uintptr_t>(q->codes) | reinterpret_cast<uintptr_t>(q->scales) | reinterpret_cast<uintptr_t>(q->zeros);
  if (bits & 15) return RT3D_ERR_INVALID_ARG;
  if (ceil_div64(q->m, 16) * ceil_div64(q->k, 64) >= (int64_t(1) << 31)) return RT3D_ERR_UNSUPPORTED;
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
bool blocks_for(long long threads, int per_block, unsigned* blocks) {
  const long long n = (threads + per_block - 1) / per_block;
  *blocks = unsigned(n);
  return n < (1ll << 31);
}

template <typename T>
rt3d_status quantize(const T* w, int64_t pitch, const rt3d_w4* q, cudaStream_t st) {
  const int n_groups = ceil_div(q->k, q->group), k_blocks = ceil_div(q->k, 64);
  const long long total = (long long)ceil_div(q->m, 16) * 16 * n_groups;
  unsigned blocks;
  if (!blocks_for(total, 128, &blocks)) return RT3D_ERR_UNSUPPORTED;
  LaunchSetup ls(dim3(blocks), dim3(128), 0, st);
  return launched(cudaLaunchKernelEx(&ls.cfg, w4_quantize_kernel<T>, w, (long long)pitch, q->m, q->k, q->group, n_groups, k_blocks,
                                     reinterpret_cast<uint32_t*>(q->codes), q->scales, q->zeros, total));
}
template <typename T>
rt3d_status unpack(const rt3d_w4* q, T* w, int64_t pitch, cudaStream_t st) {
  const int n_groups = ceil_div(q->k, q->group), k_blocks = ceil_div(q->k, 64), words = ceil_div(q->k, 8);
  const long long total = (long long)q->m * words;
  unsigned blocks;
  if (!blocks_for(total, 256, &blocks)) return RT3D_ERR_UNSUPPORTED;
  LaunchSetup ls(dim3(blocks), dim3(256), 0, st);
  return launched(cudaLaunchKernelEx(&ls.cfg, w4_unpack_kernel<T>, reinterpret_cast<const uint32_t*>(q->codes), q->scales, q->zeros, q->m,
                                     q->k, q->group, n_groups, k_blocks, words, w, (long long)pitch, total));
}
template <typename T, int kTiles, int kRows8>
rt3d_status launch_linear(const LinearArgs& a, bool fine, int ranks, cudaStream_t st) {
  const dim3 grid(unsigned(ceil_div(a.n_tiles, kTiles) * ranks), unsigned(ceil_div(a.rows, kRows8 * 8)));
  LaunchSetup ls(grid, dim3(kLinearThreads), 0, st, unsigned(ranks));
  const auto kernel = a.zeros ? (fine ? linear_w4_kernel<T, kTiles, kRows8, true, true> : linear_w4_kernel<T, kTiles, kRows8, false, true>)
                              : (fine ? linear_w4_kernel<T, kTiles, kRows8, true, false> : linear_w4_kernel<T, kTiles, kRows8, false, false>);
  return launched(cudaLaunchKernelEx(&ls.cfg, kernel, a));
}
template <typename T>
rt3d_status linear(const rt3d_tensor* x, const rt3d_w4* q, const float* bias, int relu, rt3d_tensor* y, long long rows, int sms, cudaStream_t st) {
  LinearArgs a;
  a.codes = reinterpret_cast<const uint4*>(q->codes);
  a.scales = q->scales; a.zeros = q->zeros; a.bias = bias; a.x = x->data; a.y = y->data;
  a.x_pitch = x->c_stride; a.y_pitch = y->c_stride;
  a.m = q->m; a.k = q->k; a.group_shift = q->group == 128 ? 1 : 0; a.n_groups = ceil_div(q->k, q->group);
  a.k_blocks = ceil_div(q->k, 64); a.n_tiles = ceil_div(q->m, 16); a.relu = relu ? 1 : 0; a.rows = int(rows);
  // fp32 rows take three times the registers: 16 at a time at most, in two tiles
  constexpr bool kWide = sizeof(T) == 2;
  const int rows8 = rows <= 8 ? 1 : rows <= 16 || !kWide ? 2 : 4;
  // Four tiles to a CTA (a quarter of the reads of x) where two CTAs an SM are left, inputs cut over a cluster or not;
  // then inputs are cut until there are two CTAs an SM, or every warp has one block.
  const int most_ranks = a.k_blocks >= 64 ? 8 : a.k_blocks >= 32 ? 4 : a.k_blocks >= 16 ? 2 : 1;
  const long long row_sets = ceil_div64(rows, rows8 * 8);
  int tiles = rows8 == 4 || (rows8 == 2 && !kWide) ? 2 : 4;
  while (tiles > 1 && ceil_div(a.n_tiles, tiles) * row_sets * most_ranks < 2 * sms) tiles /= 2;
  int ranks = 1;
  while (ranks < most_ranks && ceil_div(a.n_tiles, tiles) * row_sets * ranks < 2 * sms) ranks *= 2;
  const bool fine = q->group == 32;
  if (rows8 == 1)
    return tiles == 4 ? launch_linear<T, 4, 1>(a, fine, ranks, st) : tiles == 2 ? launch_linear<T, 2, 1>(a, fine, ranks, st)
                                                                                : launch_linear<T, 1, 1>(a, fine, ranks, st);
  if constexpr (kWide) {
    if (rows8 == 4) return tiles == 2 ? launch_linear<T, 2, 4>(a, fine, ranks, st) : launch_linear<T, 1, 4>(a, fine, ranks, st);
    if (tiles == 4) return launch_linear<T, 4, 2>(a, fine, ranks, st);
  }
  return tiles == 2 ? launch_linear<T, 2, 2>(a, fine, ranks, st) : launch_linear<T, 1, 2>(a, fine, ranks, st);
}

}  // namespace
}  // namespace rt3d

using namespace rt3d;

extern "C" {

int64_t rt3d_w4_codes_bytes(int m, int k) {
  if (!valid_extents(m, k) || ceil_div64(m, 16) * ceil_div64(k, 64) >= (int64_t(1) << 31)) return -1;
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
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return dtype == RT3D_BF16 ? quantize(static_cast<const __nv_bfloat16*>(w), pitch, q, st) : quantize(static_cast<const float*>(w), pitch, q, st);
}

rt3d_status rt3d_w4_unpack(const rt3d_w4* q, int dtype, void* w, int64_t pitch, void* stream) {
  const rt3d_status s = check_matrix(w, dtype, pitch, q);
  if (s != RT3D_OK) return s;
  if (plan_only()) return RT3D_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return dtype == RT3D_BF16 ? unpack(q, static_cast<__nv_bfloat16*>(w), pitch, st) : unpack(q, static_cast<float*>(w), pitch, st);
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
  return x->dtype == RT3D_BF16 ? linear<__nv_bfloat16>(x, q, bias, relu, y, rows, dev.sm_count, st)
                               : linear<float>(x, q, bias, relu, y, rows, dev.sm_count, st);
}

}  // extern "C"
