// Products of many rows with 4-bit weights, on tcgen05.
//
// As in w4.cu a group's sum of (c - z) x is exact but for the fp32 additions, and its scale multiplies it in fp32: so every group has
// an accumulator of its own in tensor memory, which the warps for the results drain into registers, times the scale of their filter,
// while the next groups' products run.  128 filters are the products' rows (TMEM lanes: a thread has one filter, whose scale is
// one number), kCols rows of x their columns.  Eight warps turn codes into the bf16 operand (c - z) / 64 in shared memory, 128 filters x
// 64 inputs a stage; x comes by TMA, which also makes zeros of what lies behind the last input and row.
// A stage of 128 filters x 128 inputs x 128 rows writes 64 KB of shared memory and reads 64 KB, 1024 clocks at 128 bytes a clock, against 512
// of the tensor cores; it takes 1650, the hand-overs between the warps (4096 x 8192, groups of 128: 64 rows 14 us, 128 rows 18, 256 rows 29,
// 0.82 TB/s and 600 TFLOP/s; with groups of 32, four sums to a stage, 75).  fp32 rows, bound by the warps that split them: 64 rows 26 us, with
// groups of 32 38, 512 rows 240.
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>
#include <cstring>
#include <type_traits>

#include "pdl.cuh"
#include "rt3d.h"
#include "rt3d_internal.h"
#include "umma_common.cuh"
#include "w4.cuh"

namespace rt3d {

CUresult encode_tiled(CUtensorMap* map, CUtensorMapDataType type, cuuint32_t rank, void* data, const cuuint64_t* dims, const cuuint64_t* strides,
                      const cuuint32_t* box, const cuuint32_t* steps, CUtensorMapSwizzle swizzle);      // api.cu

namespace {

constexpr int kCodeWarps = 8;
constexpr int kMine = 32;                            // columns of a thread for the results
constexpr int kSums = 4;                             // accumulators in tensor memory
constexpr uint32_t kFilterBytes = 128 * 128;         // 128 filters x 64 bf16
constexpr int kAhead = 4;                            // stages of codes on their way to a warp

struct ManyBars {
  Barriers b;                                        // full, empty: the ring
  unsigned long long sum_full[kSums], sum_empty[kSums];
};

// Of bf16 rows one operand, by TMA; fp32 rows are split into three bf16 parts that add up to the value by warps of their own (w4.cuh).
template <int kCols, bool kFloat>
struct ManyShape {
  static constexpr int kParts = kFloat ? 3 : 1, kRowWarps = kFloat ? 8 : 0;
  // 128 inputs: two blocks of filters, two of rows.  (A stage of 64 left the thread that issues the products 1200 clocks a stage, twice
  // what they take: 4096 x 8192, 256 rows, 41 us.)
  static constexpr uint32_t kRowsAt = 2 * kFilterBytes, kPartBytes = 2 * kCols * 128, kStage = kRowsAt + kParts * kPartBytes;
  static constexpr int kRing = kFloat ? 2 : kCols == 64 ? 4 : 3;
  static constexpr int kResultWarps = 4 * kCols / kMine, kThreads = 32 * (2 + kResultWarps + kCodeWarps + kRowWarps);
  static constexpr uint32_t kSumBytes = 128 * kCols * 4, kBytes = kRing * kStage + 1024 + sizeof(ManyBars);
  static_assert(kSumBytes <= kRing * kStage, "the sums go where the ring was");
};

// kShift: log2 of the 16s of inputs in a group.
template <int kCols, bool kFloat, bool kZeros, int kShift>
__global__ void __launch_bounds__((ManyShape<kCols, kFloat>::kThreads), 1)
linear_w4_many_kernel(const __grid_constant__ CUtensorMap xmap, const LinearArgs a, int splits, int32_t* __restrict__ err) {
  typedef ManyShape<kCols, kFloat> S;
  typedef typename std::conditional<kFloat, float, __nv_bfloat16>::type T;
  constexpr int kResultWarps = S::kResultWarps;
  extern __shared__ unsigned char smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  unsigned char* ring = smem_raw + (base - smem_u32(smem_raw));
  ManyBars* mb = reinterpret_cast<ManyBars*>(ring + S::kRing * S::kStage);
  Barriers* bars = &mb->b;
  const int warp = uniform(int(threadIdx.x >> 5)), lane = threadIdx.x & 31;
  const int split = splits > 1 ? int(cluster_ctarank()) : 0;
  const int filter0 = int(blockIdx.x) / splits * 128;
  const long long row0 = (long long)blockIdx.y * kCols;
  // stages of 128 inputs, in which no group is cut
  const int pairs = (a.k_blocks + 1) / 2;
  const int p_first = int((long long)pairs * split / splits), p_last = int((long long)pairs * (split + 1) / splits);
  constexpr int kGroup16 = 1 << kShift, kGroups = 8 >> kShift;      // 16s in a group, groups in a stage
  const int n_sums = (p_last - p_first) * kGroups;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kRing; ++s) { mbar_init(smem_u32(&bars->full[s]), kFloat ? S::kRowWarps + kCodeWarps : 1 + kCodeWarps); mbar_init(smem_u32(&bars->empty[s]), 1); }
    for (int q = 0; q < kSums; ++q) { mbar_init(smem_u32(&mb->sum_full[q]), 1); mbar_init(smem_u32(&mb->sum_empty[q]), kResultWarps); }
    bars->abort_flag = 0;
    bars->wait_limit = kWaitCycles;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    if (!kFloat) tma_prefetch_map(&xmap);
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(smem_u32(&bars->tmem_base)), "r"(uint32_t(kSums * kCols)) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = uniform(uint32_t(bars->tmem_base));
  pdl_launch();
  pdl_wait();

  if (warp == 0) {
    // ------------------------------------------------------------------ rows of x
    if (!kFloat && lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      for (int p = p_first; p < p_last; ++p) {
        const uint32_t full = smem_u32(&bars->full[stage]), to = base + stage * S::kStage + S::kRowsAt;
        if (!mbar_wait(smem_u32(&bars->empty[stage]), phase ^ 1u, bars, err, 1)) break;
        mbar_expect_tx(full, uint32_t(kCols) * 256);
        tma_load_2d(to, &xmap, full, p * 128, int(row0));
        tma_load_2d(to + kCols * 128, &xmap, full, p * 128 + 64, int(row0));
        if (++stage == S::kRing) { stage = 0; phase ^= 1u; }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ products
    const bool elected = elect_one();
    const uint32_t idesc = instr_desc_bf16(kCols);
    int stage = 0;
    uint32_t phase = 0, sum = 0;
    bool ok = true;
    for (int p = p_first; p < p_last && ok; ++p) {
      if (!mbar_wait_warp(smem_u32(&bars->full[stage]), phase, bars, err, 2)) break;
      tc_fence_after();
      const uint32_t at = base + stage * S::kStage;
      const uint64_t filters = smem_desc_sw128(at), rows = smem_desc_sw128(at + S::kRowsAt);
#pragma unroll
      for (int g = 0; g < kGroups; ++g, ++sum) {
        const uint32_t buf = sum % kSums;
        if (!mbar_wait_warp(smem_u32(&mb->sum_empty[buf]), ((sum / kSums) & 1u) ^ 1u, bars, err, 3)) { ok = false; break; }
        tc_fence_after();
        if (elected) {
#pragma unroll
          for (int i = 0; i < kGroup16; ++i) {
            const int k = g * kGroup16 + i;          // of the stage's eight 16s
#pragma unroll
            for (int part = S::kParts - 1; part >= 0; --part)                // the smallest parts first
              umma_bf16(tmem + buf * kCols, filters + (k >> 2) * (kFilterBytes >> 4) + 2 * (k & 3),
                        rows + part * (S::kPartBytes >> 4) + (k >> 2) * (kCols * 128 >> 4) + 2 * (k & 3), idesc, i || part < S::kParts - 1 ? 1u : 0u);
          }
          umma_commit(smem_u32(&mb->sum_full[buf]));
        }
      }
      if (ok && elected) umma_commit(smem_u32(&bars->empty[stage]));
      if (++stage == S::kRing) { stage = 0; phase ^= 1u; }
    }
    __syncwarp();
  } else if (warp < 2 + kResultWarps) {
    // ------------------------------------------------------------------ results
    const int quad = warp & 3, half = (warp - 2) >> 2, filter = quad * 32 + lane;
    const int tile = min((filter0 + filter) >> 4, a.n_tiles - 1);
    const uint16_t* scales = a.scales + (long long)tile * a.n_groups * 16 + (filter & 15);
    const int g0 = p_first * kGroups;
    float acc[kMine];
#pragma unroll
    for (int q = 0; q < kMine; ++q) acc[q] = 0.f;
    // scales are asked for eight groups ahead: one ahead, every group waited 900 clocks for the next one's
    constexpr int kScales = 8;
    uint16_t scale[kScales];
    auto scale_of = [&](int n) { return __ldg(scales + (long long)min(g0 + n, a.n_groups - 1) * 16); };
#pragma unroll
    for (int q = 0; q < kScales; ++q) scale[q] = scale_of(q);
    bool ok = true;
    for (int n0 = 0; n0 < n_sums && ok; n0 += kScales) {
#pragma unroll
      for (int q = 0; q < kScales; ++q) {
        const int n = n0 + q, buf = n % kSums;
        if (n >= n_sums) break;
        const float s = bf16_float(scale[q]);
        scale[q] = scale_of(n + kScales);
        if (!mbar_wait_warp(smem_u32(&mb->sum_full[buf]), uint32_t(n / kSums) & 1u, bars, err, 4)) { ok = false; break; }
        tc_fence_after();
        const uint32_t at = tmem + (uint32_t(quad * 32) << 16) + buf * kCols + half * kMine;
        uint32_t r[32];
        tmem_ld32(at, r);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&mb->sum_empty[buf]));
#pragma unroll
        for (int e = 0; e < 32; ++e) acc[e] = fmaf(s, __uint_as_float(r[e]), acc[e]);
      }
    }
    const int i = filter0 + filter;
    T* y = static_cast<T*>(a.y);
    if (splits == 1) {
      if (!bars->abort_flag && i < a.m) {
        const float bias = a.bias ? __ldg(a.bias + i) : 0.f;
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
          const long long r = row0 + half * kMine + q;
          const float v = acc[q] * 64.f + bias;
          if (r < a.rows) store_value(y + r * a.y_pitch + i, a.relu ? relu_of(v) : v);
        }
      }
    } else {
      // [column][filter], where the ring was: its copies have all been read
      float* part = reinterpret_cast<float*>(ring);
#pragma unroll
      for (int q = 0; q < kMine; ++q) part[(half * kMine + q) * 128 + filter] = acc[q];
      __syncwarp();
      cluster_sync_all();
      if (!bars->abort_flag && i < a.m) {
        const float bias = a.bias ? __ldg(a.bias + i) : 0.f;
        for (int c = split * kCols / splits + half; c < (split + 1) * kCols / splits; c += kResultWarps / 4) {
          float v = 0.f;
          for (int q = 0; q < splits; ++q) v += ld_cluster_f32(mapa_shared(base + (c * 128 + filter) * 4, uint32_t(q)));
          v = v * 64.f + bias;
          if (row0 + c < a.rows) store_value(y + (row0 + c) * a.y_pitch + i, a.relu ? relu_of(v) : v);
        }
      }
    }
  } else if (warp < 2 + kResultWarps + kCodeWarps) {
    // ------------------------------------------------------------------ codes: a tile of 16 filters for each warp
    const int w = warp - 2 - kResultWarps, g = lane >> 2, t = lane & 3;
    const int tile = min((filter0 >> 4) + w, a.n_tiles - 1);
    // places of filter g: units t and 4 + t of its row of 128 bytes, swizzled; filter g + 8 lies 1024 bytes further.  Odd filters write
    // the second unit first: eight lanes' 16 bytes then lie in eight columns.
    const int odd = g & 1;
    const uint32_t row = uint32_t(w * 16 + g) * 128, at0 = row + (((t + 4 * odd) ^ g) << 4), at1 = row + (((t + 4 * (odd ^ 1)) ^ g) << 4);
    // Words and zero points come in the order in which they are written.
    const uint2* codes = reinterpret_cast<const uint2*>(a.codes + ((long long)tile * a.k_blocks) * 32 + lane) + odd;
    const int other = odd ? -1 : 1;                  // from the unit written first to the second
    const uint8_t* zeros = kZeros ? a.zeros + (long long)tile * a.n_groups * 16 + g : nullptr;
    constexpr int kZ = kShift > 1 ? 1 : 2;           // zero points of a block: one for both halves, or one each
    uint2 words[kAhead][2][2] = {};                  // block, unit (filters g and g + 8); of a block that is not there: anything, as x is zero there
    uint32_t z[kAhead][2][kZ] = {};                  // of both filters
    auto fetch = [&](int slot, int p) {
      if (p >= p_last) return;
#pragma unroll
      for (int d = 0; d < 2; ++d) {
        const int b = 2 * p + d;
        if (b >= a.k_blocks) continue;
        const uint2* src = codes + (long long)b * 64;
        words[slot][d][0] = __ldg(src); words[slot][d][1] = __ldg(src + other);
        if (kZeros && (d == 0 || kShift < 3)) {
#pragma unroll
          for (int h = 0; h < kZ; ++h) {
            const int grp = kShift == 1 ? min(b * 2 + (h ^ odd), a.n_groups - 1) : kShift == 2 ? b : p;
            z[slot][d][h] = __ldg(zeros + grp * 16) | uint32_t(__ldg(zeros + grp * 16 + 8)) << 16;
          }
        }
      }
    };
#pragma unroll
    for (int q = 0; q < kAhead; ++q) fetch(q, p_first + q);
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int p0 = p_first; p0 < p_last && ok; p0 += kAhead) {
#pragma unroll
      for (int q = 0; q < kAhead; ++q) {
        if (p0 + q >= p_last) break;
        if (!mbar_wait_warp(smem_u32(&bars->empty[stage]), phase ^ 1u, bars, err, 5)) { ok = false; break; }
        const uint32_t to = base + stage * S::kStage;
        uint32_t minus[2] = {kMinusEighth, kMinusEighth};
#pragma unroll
        for (int d = 0; d < 2; ++d)
#pragma unroll
          for (int n = 0; n < 2; ++n) {
            if (kZeros && n < kZ && (d == 0 || kShift < 3)) {
              minus[0] = minus_zero(z[q][d][n < kZ ? n : 0] & 0xffffu);
              minus[1] = minus_zero(z[q][d][n < kZ ? n : 0] >> 16);
            }
#pragma unroll
            for (int f = 0; f < 2; ++f) {
              uint32_t v[4];
              spread_codes(f ? words[q][d][n].y : words[q][d][n].x, minus[f], v);
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + d * kFilterBytes + (n ? at1 : at0) + f * 1024), "r"(v[0]), "r"(v[1]),
                           "r"(v[2]), "r"(v[3]) : "memory");
            }
          }
        fetch(q, p0 + q + kAhead);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars->full[stage]));
        if (++stage == S::kRing) { stage = 0; phase ^= 1u; }
      }
    }
  }
  else if constexpr (kFloat) {
    // ------------------------------------------------------------------ fp32 rows: every warp has each eighth row
    const int w = warp - 2 - kResultWarps - kCodeWarps, g = lane >> 2, t = lane & 3, r = w * (kCols / S::kRowWarps) + g, odd = r & 1;
    static_assert(kCols == 8 * S::kRowWarps, "a row for each four lanes");
    const float* x = row0 + r < a.rows ? static_cast<const float*>(a.x) + (row0 + r) * a.x_pitch : nullptr;
    // as the filters' units: the two halves of a block in the order that keeps eight lanes' 16 bytes apart
    const uint32_t to0 = uint32_t(r) * 128 + (((t + 4 * odd) ^ (r & 7)) << 4), to1 = uint32_t(r) * 128 + (((t + 4 * (odd ^ 1)) ^ (r & 7)) << 4);
    float4 v[2][2][2];                               // block, unit, half of it: a stage ahead
    auto fetch = [&](int p) {
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int k0 = p * 128 + d * 64 + (n ^ odd) * 32 + t * 8;
          v[d][n][0] = v[d][n][1] = make_float4(0.f, 0.f, 0.f, 0.f);
          if (!x || p >= p_last || k0 >= a.k) continue;
          if (k0 + 8 <= a.k) {
            v[d][n][0] = __ldg(reinterpret_cast<const float4*>(x + k0)); v[d][n][1] = __ldg(reinterpret_cast<const float4*>(x + k0 + 4));
          } else {
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = k0 + e < a.k ? __ldg(x + k0 + e) : 0.f;
            v[d][n][0] = make_float4(f[0], f[1], f[2], f[3]); v[d][n][1] = make_float4(f[4], f[5], f[6], f[7]);
          }
        }
    };
    fetch(p_first);
    int stage = 0;
    uint32_t phase = 0;
    for (int p = p_first; p < p_last; ++p) {
      if (!mbar_wait_warp(smem_u32(&bars->empty[stage]), phase ^ 1u, bars, err, 6)) break;
      const uint32_t to = base + stage * S::kStage + S::kRowsAt;
#pragma unroll
      for (int d = 0; d < 2; ++d)
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          uint32_t part[3][4];
          const float f[8] = {v[d][n][0].x, v[d][n][0].y, v[d][n][0].z, v[d][n][0].w, v[d][n][1].x, v[d][n][1].y, v[d][n][1].z, v[d][n][1].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) split_pair(f[2 * e], f[2 * e + 1], part[0][e], part[1][e], part[2][e]);
#pragma unroll
          for (int q = 0; q < 3; ++q)
            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to + q * S::kPartBytes + d * (kCols * 128) + (n ? to1 : to0)), "r"(part[q][0]),
                         "r"(part[q][1]), "r"(part[q][2]), "r"(part[q][3]) : "memory");
        }
      fetch(p + 1);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars->full[stage]));
      if (++stage == S::kRing) { stage = 0; phase ^= 1u; }
    }
  }
  if (splits > 1) {
    __syncwarp();
    if (warp < 2 || warp >= 2 + kResultWarps) cluster_sync_all();
    cluster_sync_all();                              // nobody leaves while its sums are still being read
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
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(uint32_t(kSums * kCols)) : "memory");
  }
}

template <int kCols, bool kFloat>
rt3d_status launch_many(const LinearArgs& a, const DeviceInfo& dev, cudaStream_t st) {
  typedef ManyShape<kCols, kFloat> S;
  CUtensorMap xmap;
  std::memset(&xmap, 0, sizeof(xmap));
  const cuuint64_t dims[2] = {cuuint64_t(a.k), cuuint64_t(a.rows)}, strides[1] = {cuuint64_t(a.x_pitch) * 2};
  const cuuint32_t box[2] = {64, kCols}, estr[2] = {1, 1};
  if (!kFloat && encode_tiled(&xmap, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(a.x), dims, strides, box, estr, CU_TENSOR_MAP_SWIZZLE_128B) != CUDA_SUCCESS)
    return RT3D_ERR_CUDA;
  typedef void (*Kernel)(CUtensorMap, LinearArgs, int, int32_t*);
  static const Kernel kernels[2][3] = {{linear_w4_many_kernel<kCols, kFloat, false, 1>, linear_w4_many_kernel<kCols, kFloat, false, 2>, linear_w4_many_kernel<kCols, kFloat, false, 3>},
                                       {linear_w4_many_kernel<kCols, kFloat, true, 1>, linear_w4_many_kernel<kCols, kFloat, true, 2>, linear_w4_many_kernel<kCols, kFloat, true, 3>}};
  const int kind = a.fine ? 0 : a.group_shift + 1;
  const Kernel kernel = kernels[a.zeros != nullptr][kind];
  static std::atomic<bool> attr_done[kMaxDevices][2][3];
  const int d = current_device_index();
  if (d < 0) return RT3D_ERR_CUDA;
  std::atomic<bool>& done = attr_done[d][a.zeros != nullptr][kind];
  if (!done.load()) {
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(S::kBytes)) != cudaSuccess) return RT3D_ERR_CUDA;
    done.store(true);
  }
  const int tiles = ceil_div(a.n_tiles, 8);
  const long long row_tiles = ceil_div64(a.rows, kCols);
  // the inputs are shared out while that fills SMs and leaves every CTA eight blocks
  int splits = 1;
  while (splits < 8 && tiles * row_tiles * splits * 2 <= dev.sm_count && a.k_blocks >= 16 * splits) splits *= 2;
  LaunchSetup ls(dim3(unsigned(tiles * splits), unsigned(row_tiles)), dim3(S::kThreads), S::kBytes, st, unsigned(splits));
  if (cudaLaunchKernelEx(&ls.cfg, kernel, xmap, a, splits, dev.err) != cudaSuccess) return RT3D_ERR_CUDA;
  count_launches(1);
  return RT3D_OK;
}

}  // namespace

rt3d_status linear_w4_many_rows(const LinearArgs& a, int dtype, const DeviceInfo& dev, cudaStream_t st) {
  if (dtype == RT3D_F32) return launch_many<64, true>(a, dev, st);
  return a.rows <= 64 ? launch_many<64, false>(a, dev, st) : launch_many<128, false>(a, dev, st);
}

}  // namespace rt3d
