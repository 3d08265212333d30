// 4-bit weights with group scales: quantisation, its inverse and the products with a few rows of activations.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "pdl.cuh"
#include "rt3d.h"
#include "rt3d_internal.h"

namespace rt3d {
namespace {

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

// One warp for an output: lanes take words of eight inputs.
template <typename T>
__global__ void linear_w4_kernel(const T* __restrict__ x, long long x_pitch, const uint32_t* __restrict__ codes,
                                 const uint16_t* __restrict__ scales, const uint8_t* __restrict__ zeros, int m, int k, int group,
                                 int n_groups, int k_blocks, const float* __restrict__ bias, int relu, T* __restrict__ y,
                                 long long y_pitch, long long total) {
  pdl_entry();
  const long long out = ((long long)blockIdx.x * blockDim.x + threadIdx.x) >> 5;
  if (out >= total) return;
  const int lane = threadIdx.x & 31, i = int(out % m);
  const long long row = out / m;
  float sum = 0.f;
  for (int kw = lane; kw * 8 < k; kw += 32) {
    const long long at = ((long long)(i >> 4) * n_groups + kw * 8 / group) * 16 + (i & 15);
    const float s = bf16_float(scales[at]), z = zeros ? float(zeros[at]) : 8.f;
    const uint32_t word = codes[word_of(i, kw, k_blocks)];
    float part = 0.f;
    for (int e = 0; e < 8 && kw * 8 + e < k; ++e)
      part += (float((word >> shift_of(e)) & 15u) - z) * value_of(x + row * x_pitch + kw * 8 + e);
    sum += s * part;
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if (lane == 0) {
    if (bias) sum += bias[i];
    store_value(y + row * y_pitch + i, relu ? fmaxf(sum, 0.f) : sum);
  }
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
template <typename T>
rt3d_status linear(const rt3d_tensor* x, const rt3d_w4* q, const float* bias, int relu, rt3d_tensor* y, long long rows, cudaStream_t st) {
  const int n_groups = ceil_div(q->k, q->group), k_blocks = ceil_div(q->k, 64);
  const long long total = rows * q->m;
  unsigned blocks;
  if (!blocks_for(total * 32, 256, &blocks)) return RT3D_ERR_UNSUPPORTED;
  LaunchSetup ls(dim3(blocks), dim3(256), 0, st);
  return launched(cudaLaunchKernelEx(&ls.cfg, linear_w4_kernel<T>, static_cast<const T*>(x->data), (long long)x->c_stride,
                                     reinterpret_cast<const uint32_t*>(q->codes), q->scales, q->zeros, q->m, q->k, q->group, n_groups,
                                     k_blocks, bias, relu ? 1 : 0, static_cast<T*>(y->data), (long long)y->c_stride, total));
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
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return x->dtype == RT3D_BF16 ? linear<__nv_bfloat16>(x, q, bias, relu, y, rows, st) : linear<float>(x, q, bias, relu, y, rows, st);
}

}  // extern "C"
