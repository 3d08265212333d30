// Orthogonalised updates: Newton-Schulz products of a layer's gradient, and the optimiser step around them.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>

#include "pdl.cuh"
#include "rt3d.h"
#include "rt3d_internal.h"

namespace rt3d {
namespace {

constexpr int kNormBlocks = 512;

__device__ __forceinline__ float value_of(const float* p) { return *p; }
__device__ __forceinline__ float value_of(const __nv_bfloat16* p) { return __bfloat162float(*p); }

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
template <typename T, bool kFirst>
__device__ __forceinline__ float source_value(const Source<T>& s, int i, int j, int k) {
  if (!s.momentum) return value_of(s.g + (long long)i * s.pitch + j);
  const long long at = (long long)i * k + j;
  const bool keep = !s.mask || s.mask[at];
  float v = s.momentum[at];
  const float g = value_of(s.g + at);
  if (kFirst) {
    v = keep ? fmaf(s.mu, v, g) : 0.f;
    s.momentum[at] = v;
  }
  return !keep ? 0.f : s.nesterov ? fmaf(s.mu, v, g) : v;
}

// Sums of squares of the blocks' shares, in 64 bits: neither overflow nor the order of a long sum matters.
template <typename T>
__global__ void __launch_bounds__(256)
square_sums_kernel(Source<T> s, int m, int k, double* __restrict__ sums) {
  pdl_entry();
  __shared__ double part[8];
  double sum = 0.0;
  for (long long idx = (long long)blockIdx.x * 256 + threadIdx.x; idx < (long long)m * k; idx += (long long)gridDim.x * 256) {
    const float v = source_value<T, true>(s, int(idx / k), int(idx % k), k);
    sum += double(v) * v;
  }
  for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < 8; ++w) sum += part[w];
    sums[blockIdx.x] = sum;
  }
}

// X = the source over its norm, transposed where there are more rows than columns.
template <typename T>
__global__ void __launch_bounds__(256)
normalise_kernel(Source<T> s, int m, int k, const double* __restrict__ sums, double eps, float* __restrict__ x) {
  pdl_entry();
  double sum = 0.0;
  for (int b = 0; b < kNormBlocks; ++b) sum += sums[b];
  const double inv = 1.0 / (sqrt(sum) + eps);
  for (long long idx = (long long)blockIdx.x * 256 + threadIdx.x; idx < (long long)m * k; idx += (long long)gridDim.x * 256) {
    const int i = int(idx / k), j = int(idx % k);
    x[m > k ? (long long)j * m + i : idx] = float(source_value<T, false>(s, i, j, k) * inv);
  }
}

// C[i][j] = alpha sum_l A[i][l] B[l][j] + beta D[i][j]; strides of B given, the others row-major.
__global__ void __launch_bounds__(256)
product_kernel(const float* __restrict__ a, long long lda, const float* __restrict__ b, long long b_row, long long b_col, int m, int n,
               int k, float alpha, const float* __restrict__ d, float beta, float* __restrict__ c, long long ldc) {
  pdl_entry();
  __shared__ float as[16][65], bs[16][65];
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, ti = threadIdx.x / 16, tj = threadIdx.x % 16;
  float acc[4][4] = {};
  for (int l0 = 0; l0 < k; l0 += 16) {
    for (int q = threadIdx.x; q < 1024; q += 256) {
      const int l = q % 16, r = q / 16;
      as[l][r] = i0 + r < m && l0 + l < k ? a[(i0 + r) * lda + l0 + l] : 0.f;
      const int bl = b_row == 1 ? l : q / 64, bj = b_row == 1 ? r : q % 64;
      bs[bl][bj] = j0 + bj < n && l0 + bl < k ? b[(l0 + bl) * b_row + (j0 + bj) * b_col] : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int l = 0; l < 16; ++l)
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[p][q] = fmaf(as[l][ti + 16 * p], bs[l][tj + 16 * q], acc[p][q]);
    __syncthreads();
  }
  for (int p = 0; p < 4; ++p)
    for (int q = 0; q < 4; ++q) {
      const int i = i0 + ti + 16 * p, j = j0 + tj + 16 * q;
      if (i < m && j < n) c[i * ldc + j] = alpha * acc[p][q] + (d ? beta * d[i * ldc + j] : 0.f);
    }
}

__global__ void direction_out_kernel(const float* __restrict__ x, int m, int k, __nv_bfloat16* __restrict__ out, long long pitch) {
  pdl_entry();
  for (long long idx = (long long)blockIdx.x * 256 + threadIdx.x; idx < (long long)m * k; idx += (long long)gridDim.x * 256) {
    const int i = int(idx / k), j = int(idx % k);
    out[i * pitch + j] = __float2bfloat16_rn(x[m > k ? (long long)j * m + i : idx]);
  }
}
__global__ void apply_kernel(const float* __restrict__ x, int m, int k, const uint8_t* __restrict__ mask, float keep_share, float step,
                             float* __restrict__ w) {
  pdl_entry();
  for (long long idx = (long long)blockIdx.x * 256 + threadIdx.x; idx < (long long)m * k; idx += (long long)gridDim.x * 256) {
    const int i = int(idx / k), j = int(idx % k);
    const float o = x[m > k ? (long long)j * m + i : idx];
    w[idx] = !mask || mask[idx] ? fmaf(-step, o, keep_share * w[idx]) : 0.f;
  }
}

constexpr int kMostSteps = 16;
struct Plan {
  int steps;
  double eps;
  float abc[kMostSteps][3];
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
    if (!(top <= 1.9) || !(most_p <= 50.0)) return RT3D_ERR_UNSUPPORTED;
  }
  return RT3D_OK;
}

struct Workspace {
  double* sums;
  float *x, *y, *gram, *poly;
};
int64_t workspace_of(int m, int k, char* base, Workspace* ws) {
  int64_t at = 0;
  auto take = [&](int64_t bytes) {
    char* p = base + at;
    at += (bytes + 255) / 256 * 256;
    return p;
  };
  const int64_t small = m < k ? m : k, size = int64_t(m) * k;
  Workspace w;
  w.sums = reinterpret_cast<double*>(take(kNormBlocks * 8));
  w.x = reinterpret_cast<float*>(take(size * 4));
  w.y = reinterpret_cast<float*>(take(size * 4));
  w.gram = reinterpret_cast<float*>(take(small * small * 4));
  w.poly = reinterpret_cast<float*>(take(small * small * 4));
  if (ws) *ws = w;
  return at;
}

rt3d_status launched(cudaError_t e) {
  if (e != cudaSuccess) return RT3D_ERR_CUDA;
  count_launches(1);
  return RT3D_OK;
}

rt3d_status product(const float* a, long long lda, const float* b, long long b_row, long long b_col, int m, int n, int k, float alpha,
                    const float* d, float beta, float* c, long long ldc, cudaStream_t st) {
  LaunchSetup ls(dim3(unsigned(ceil_div(n, 64)), unsigned(ceil_div(m, 64))), dim3(256), 0, st);
  return launched(cudaLaunchKernelEx(&ls.cfg, product_kernel, a, lda, b, b_row, b_col, m, n, k, alpha, d, beta, c, ldc));
}

// X of the last step; *x is where it lies.
template <typename T>
rt3d_status direction(const Source<T>& src, int m, int k, const Plan& plan, const Workspace& ws, const float** x, cudaStream_t st) {
  LaunchSetup ls(dim3(kNormBlocks), dim3(256), 0, st);
  rt3d_status s = launched(cudaLaunchKernelEx(&ls.cfg, square_sums_kernel<T>, src, m, k, ws.sums));
  if (s != RT3D_OK) return s;
  if ((s = launched(cudaLaunchKernelEx(&ls.cfg, normalise_kernel<T>, src, m, k, (const double*)ws.sums, plan.eps, ws.x))) != RT3D_OK) return s;
  const int n = m < k ? m : k, l = m < k ? k : m;
  float *cur = ws.x, *next = ws.y;
  for (int i = 0; i < plan.steps; ++i) {
    const float* abc = plan.abc[i];
    if ((s = product(cur, l, cur, 1, l, n, n, l, 1.f, nullptr, 0.f, ws.gram, n, st)) != RT3D_OK) return s;
    if ((s = product(ws.gram, n, ws.gram, n, 1, n, n, n, abc[2], ws.gram, abc[1], ws.poly, n, st)) != RT3D_OK) return s;
    if ((s = product(ws.poly, n, cur, l, 1, n, l, n, 1.f, cur, abc[0], next, l, st)) != RT3D_OK) return s;
    float* t = cur; cur = next; next = t;
  }
  *x = cur;
  return RT3D_OK;
}

rt3d_status check_call(const void* g, int dtype, int m, int k, void* workspace, int64_t bytes) {
  if (!g || !workspace || m < 1 || k < 1 || (dtype != RT3D_F32 && dtype != RT3D_BF16)) return RT3D_ERR_INVALID_ARG;
  if (reinterpret_cast<uintptr_t>(g) % (dtype == RT3D_BF16 ? 2 : 4) || reinterpret_cast<uintptr_t>(workspace) % 16) return RT3D_ERR_INVALID_ARG;
  const int64_t need = rt3d_ortho_workspace(m, k);
  if (need < 0) return RT3D_ERR_UNSUPPORTED;
  return bytes < need ? RT3D_ERR_WORKSPACE : RT3D_OK;
}

template <typename T>
rt3d_status orthogonalize(const T* g, int64_t pitch, int m, int k, const Plan& plan, __nv_bfloat16* out, int64_t out_pitch, char* base, cudaStream_t st) {
  Workspace ws;
  workspace_of(m, k, base, &ws);
  const float* x = nullptr;
  const rt3d_status s = direction(Source<T>{g, pitch, nullptr, nullptr, 0.f, 0}, m, k, plan, ws, &x, st);
  if (s != RT3D_OK) return s;
  LaunchSetup ls(dim3(kNormBlocks), dim3(256), 0, st);
  return launched(cudaLaunchKernelEx(&ls.cfg, direction_out_kernel, x, m, k, out, (long long)out_pitch));
}

template <typename T>
rt3d_status update(float* w, float* momentum, const T* g, const uint8_t* mask, int m, int k, const rt3d_update_params& p, const Plan& plan,
                   char* base, cudaStream_t st) {
  Workspace ws;
  workspace_of(m, k, base, &ws);
  const float* x = nullptr;
  const rt3d_status s = direction(Source<T>{g, k, momentum, mask, p.mu, p.nesterov}, m, k, plan, ws, &x, st);
  if (s != RT3D_OK) return s;
  LaunchSetup ls(dim3(kNormBlocks), dim3(256), 0, st);
  return launched(cudaLaunchKernelEx(&ls.cfg, apply_kernel, x, m, k, mask, float(1.0 - double(p.lr) * p.weight_decay),
                                     float(double(p.lr) * p.scale), w));
}

}  // namespace
}  // namespace rt3d

using namespace rt3d;

extern "C" {

int64_t rt3d_ortho_workspace(int m, int k) {
  if (m < 1 || k < 1 || (m > 65535 && k > 65535)) return -1;
  return workspace_of(m, k, nullptr, nullptr);
}

rt3d_status rt3d_orthogonalize(const void* g, int dtype, int64_t g_pitch, int m, int k, const rt3d_ortho_params* p, void* out,
                               int64_t out_pitch, void* workspace, int64_t workspace_bytes, void* stream) {
  Plan plan;
  rt3d_status s = check_call(g, dtype, m, k, workspace, workspace_bytes);
  if (s != RT3D_OK) return s;
  if (!out || reinterpret_cast<uintptr_t>(out) % 2 || g_pitch < k || out_pitch < k) return RT3D_ERR_INVALID_ARG;
  const char *g0 = static_cast<const char*>(g), *o0 = static_cast<const char*>(out);
  const int64_t size = dtype == RT3D_BF16 ? 2 : 4;
  if (g0 < o0 + ((m - 1) * out_pitch + k) * 2 && o0 < g0 + ((m - 1) * g_pitch + k) * size) return RT3D_ERR_INVALID_ARG;
  if ((s = make_plan(p, &plan)) != RT3D_OK || plan_only()) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* base = static_cast<char*>(workspace);
  __nv_bfloat16* o = static_cast<__nv_bfloat16*>(out);
  return dtype == RT3D_BF16 ? orthogonalize(static_cast<const __nv_bfloat16*>(g), g_pitch, m, k, plan, o, out_pitch, base, st)
                            : orthogonalize(static_cast<const float*>(g), g_pitch, m, k, plan, o, out_pitch, base, st);
}

rt3d_status rt3d_ortho_update(float* w, float* momentum, const void* g, int dtype, const uint8_t* mask, int m, int k,
                              const rt3d_update_params* p, void* workspace, int64_t workspace_bytes, void* stream) {
  Plan plan;
  rt3d_status s = check_call(g, dtype, m, k, workspace, workspace_bytes);
  if (s != RT3D_OK) return s;
  if (!w || !momentum || !p || reinterpret_cast<uintptr_t>(w) % 4 || reinterpret_cast<uintptr_t>(momentum) % 4) return RT3D_ERR_INVALID_ARG;
  const struct { const void* at; int64_t bytes; } area[3] = {{w, 4}, {momentum, 4}, {g, dtype == RT3D_BF16 ? 2 : 4}};
  for (int i = 0; i < 3; ++i)
    for (int j = 0; j < i; ++j) {
      const char *a = static_cast<const char*>(area[i].at), *b = static_cast<const char*>(area[j].at);
      const int64_t count = int64_t(m) * k;
      if (a < b + count * area[j].bytes && b < a + count * area[i].bytes) return RT3D_ERR_INVALID_ARG;
    }
  if (!std::isfinite(p->lr) || !std::isfinite(p->mu) || !std::isfinite(p->weight_decay) || !std::isfinite(p->scale)) return RT3D_ERR_INVALID_ARG;
  if ((s = make_plan(&p->ortho, &plan)) != RT3D_OK || plan_only()) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  char* base = static_cast<char*>(workspace);
  return dtype == RT3D_BF16 ? update(w, momentum, static_cast<const __nv_bfloat16*>(g), mask, m, k, *p, plan, base, st)
                            : update(w, momentum, static_cast<const float*>(g), mask, m, k, *p, plan, base, st);
}

}  // extern "C"
