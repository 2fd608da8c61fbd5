// Group normalisation with an activation, channels last, forward and backward.
#include "kernels.h"

namespace dat {
namespace {

constexpr int kT = 256;

struct GnArgs {
  const void* x; const void* dy; const float* gamma; const float* beta; const float* mean_in; const float* rstd_in;
  void* out; float* mean; float* rstd; float* part;
  int B, P, C, G, Cg; float eps;
};

template <typename T> __device__ __forceinline__ float load1(const T* p);
template <> __device__ __forceinline__ float load1<float>(const float* p) { return *p; }
template <> __device__ __forceinline__ float load1<bf16_t>(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(bf16_t* p, float v) { *p = f2bf(v); }

__device__ __forceinline__ float gn_xhat(float x, float mean, float rstd) { return __fmul_rn(__fsub_rn(x, mean), rstd); }
__device__ __forceinline__ float gn_z(float xhat, float gamma, float beta) { return __fadd_rn(__fmul_rn(xhat, gamma), beta); }
template <int ACT> __device__ __forceinline__ float act_of(float z) {
  if (ACT == DAT_ACT_RELU) return z <= 0.0f ? 0.0f : z;      // NaN stays
  if (ACT == DAT_ACT_SILU) return z / (1.0f + expf(-z));
  return z;
}
template <int ACT> __device__ __forceinline__ float act_grad(float z, float dy) {
  if (ACT == DAT_ACT_RELU) return z > 0.0f ? dy : 0.0f;
  if (ACT == DAT_ACT_SILU) { const float s = 1.0f / (1.0f + expf(-z)); return dy * (s * (1.0f + z * (1.0f - s))); }
  return dy;
}

__device__ float block_sum(float v, float* s) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
  __syncthreads();
  return (s[0] + s[1]) + (s[2] + s[3]);
}

// One workgroup per image and group: mean, then deviations from it, then the output.
template <typename T, int ACT>
__global__ __launch_bounds__(kT) void gn_forward_kernel(GnArgs a) {
  __shared__ float s[4];
  const int b = blockIdx.x / a.G, g = blockIdx.x % a.G, n = a.P * a.Cg;
  const T* x = (const T*)a.x + (int64_t)b * a.P * a.C + g * a.Cg;
  T* y = (T*)a.out + (int64_t)b * a.P * a.C + g * a.Cg;
  float v = 0.0f;
  for (int i = threadIdx.x; i < n; i += kT) v += load1(x + (i / a.Cg) * a.C + i % a.Cg);
  const float mean = block_sum(v, s) / (float)n;
  v = 0.0f;
  for (int i = threadIdx.x; i < n; i += kT) { const float d = load1(x + (i / a.Cg) * a.C + i % a.Cg) - mean; v = fmaf(d, d, v); }
  const float rstd = __fdiv_rn(1.0f, sqrtf(block_sum(v, s) / (float)n + a.eps));
  if (threadIdx.x == 0) { a.mean[blockIdx.x] = mean; a.rstd[blockIdx.x] = rstd; }
  for (int i = threadIdx.x; i < n; i += kT) {
    const int c = g * a.Cg + i % a.Cg, e = (i / a.Cg) * a.C + i % a.Cg;
    const float z = gn_z(gn_xhat(load1(x + e), mean, rstd), a.gamma ? a.gamma[c] : 1.0f, a.beta ? a.beta[c] : 0.0f);
    store1(y + e, act_of<ACT>(z));
  }
}

// One workgroup per image and group; part[0][b][c] = sum dz, part[1][b][c] = sum dz xhat.
template <typename T, int ACT>
__global__ __launch_bounds__(kT) void gn_backward_kernel(GnArgs a) {
  __shared__ float s[4];
  const int b = blockIdx.x / a.G, g = blockIdx.x % a.G, n = a.P * a.Cg;
  const int64_t base = (int64_t)b * a.P * a.C + g * a.Cg;
  const T* x = (const T*)a.x + base;
  const T* dy = (const T*)a.dy + base;
  T* dx = (T*)a.out + base;
  const float mean = a.mean_in[blockIdx.x], rstd = a.rstd_in[blockIdx.x];
  float c1 = 0.0f, c2 = 0.0f;
  for (int k = 0; k < a.Cg; ++k) {
    const int c = g * a.Cg + k;
    const float gamma = a.gamma ? a.gamma[c] : 1.0f, beta = a.beta ? a.beta[c] : 0.0f;
    float s1 = 0.0f, s2 = 0.0f;
    for (int p = threadIdx.x; p < a.P; p += kT) {
      const float xhat = gn_xhat(load1(x + p * a.C + k), mean, rstd);
      const float dz = act_grad<ACT>(gn_z(xhat, gamma, beta), load1(dy + p * a.C + k));
      s1 += dz; s2 = fmaf(dz, xhat, s2);
    }
    s1 = block_sum(s1, s); s2 = block_sum(s2, s);
    if (threadIdx.x == 0) { a.part[(int64_t)b * a.C + c] = s1; a.part[(int64_t)(a.B + b) * a.C + c] = s2; }
    c1 = fmaf(gamma, s1, c1); c2 = fmaf(gamma, s2, c2);
  }
  c1 /= (float)n; c2 /= (float)n;
  for (int i = threadIdx.x; i < n; i += kT) {
    const int c = g * a.Cg + i % a.Cg, e = (i / a.Cg) * a.C + i % a.Cg;
    const float gamma = a.gamma ? a.gamma[c] : 1.0f, beta = a.beta ? a.beta[c] : 0.0f;
    const float xhat = gn_xhat(load1(x + e), mean, rstd);
    const float dz = act_grad<ACT>(gn_z(xhat, gamma, beta), load1(dy + e));
    store1(dx + e, rstd * (dz * gamma - c1 - xhat * c2));
  }
}

__global__ __launch_bounds__(kT) void gn_param_kernel(const float* part, int B, int C, float* dgamma, float* dbeta) {
  const int c = blockIdx.x * kT + threadIdx.x;
  if (c >= C) return;
  float s1 = 0.0f, s2 = 0.0f;
  for (int b = 0; b < B; ++b) { s1 += part[(int64_t)b * C + c]; s2 += part[(int64_t)(B + b) * C + c]; }
  dbeta[c] = s1; dgamma[c] = s2;
}

dat_status check(dat_dtype dtype, int B, int H, int W, int C, int groups) {
  if ((dtype != DAT_F32 && dtype != DAT_BF16) || B < 0 || H < 1 || W < 1 || C < 1 || groups < 1 || C % groups) return DAT_ERR_ARG;
  constexpr int64_t most = 1 << 30;
  if ((int64_t)H * W > most || (int64_t)H * W * C > most || (int64_t)B * C > most) return DAT_ERR_SHAPE;
  return DAT_OK;
}

}  // namespace
}  // namespace dat

using namespace dat;

extern "C" size_t dat_group_norm_workspace(int pass, dat_dtype dtype, int B, int H, int W, int C, int groups) {
  if (check(dtype, B, H, W, C, groups) != DAT_OK || pass != 1) return 0;
  return (size_t)B * C * 8;
}

#define DAT_GN_LAUNCH(KERNEL, act)                                                                                   \
  do {                                                                                                               \
    if (act == DAT_ACT_RELU) hipLaunchKernelGGL((KERNEL<T, DAT_ACT_RELU>), grid, dim3(kT), 0, st, a);                \
    else if (act == DAT_ACT_SILU) hipLaunchKernelGGL((KERNEL<T, DAT_ACT_SILU>), grid, dim3(kT), 0, st, a);           \
    else hipLaunchKernelGGL((KERNEL<T, DAT_ACT_NONE>), grid, dim3(kT), 0, st, a);                                    \
  } while (0)

extern "C" dat_status dat_group_norm_forward(const void* x, const float* gamma, const float* beta, dat_dtype dtype, int B, int H,
                                             int W, int C, int groups, float eps, dat_act act, void* y, float* mean, float* rstd,
                                             void* workspace, size_t workspace_bytes, void* stream) {
  const dat_status s = check(dtype, B, H, W, C, groups);
  if (s != DAT_OK) return s;
  if (!gamma != !beta || !(eps >= 0.0f) || (unsigned)act > DAT_ACT_SILU || (B > 0 && (!x || !y || !mean || !rstd))) return DAT_ERR_ARG;
  const size_t width = dtype == DAT_BF16 ? 2 : 4, need = dat_group_norm_workspace(0, dtype, B, H, W, C, groups);
  if (!aligned(x, width) || !aligned(y, width) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return DAT_ERR_ARG;
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return DAT_ERR_ARG;
  if (B == 0) return DAT_OK;
  GnArgs a{x, nullptr, gamma, beta, nullptr, nullptr, y, mean, rstd, (float*)workspace, B, H * W, C, groups, C / groups, eps};
  hipStream_t st = (hipStream_t)stream;
  const dim3 grid((unsigned)B * groups);
  if (dtype == DAT_BF16) { using T = bf16_t; DAT_GN_LAUNCH(gn_forward_kernel, act); }
  else { using T = float; DAT_GN_LAUNCH(gn_forward_kernel, act); }
  DAT_LAUNCH_CHECK();
  return DAT_OK;
}

extern "C" dat_status dat_group_norm_backward(const void* x, const void* dy, const float* gamma, const float* beta,
                                              const float* mean, const float* rstd, dat_dtype dtype, int B, int H, int W, int C,
                                              int groups, dat_act act, void* dx, float* dgamma, float* dbeta, void* workspace,
                                              size_t workspace_bytes, void* stream) {
  const dat_status s = check(dtype, B, H, W, C, groups);
  if (s != DAT_OK) return s;
  if (!gamma != !beta || !dgamma != !dbeta || (unsigned)act > DAT_ACT_SILU || (B > 0 && (!x || !dy || !dx || !mean || !rstd))) return DAT_ERR_ARG;
  const size_t width = dtype == DAT_BF16 ? 2 : 4, need = dat_group_norm_workspace(1, dtype, B, H, W, C, groups);
  if (!aligned(x, width) || !aligned(dy, width) || !aligned(dx, width) || !aligned(gamma, 4) || !aligned(beta, 4) || !aligned(mean, 4) ||
      !aligned(rstd, 4) || !aligned(dgamma, 4) || !aligned(dbeta, 4)) return DAT_ERR_ARG;
  if (need && (!workspace || workspace_bytes < need || !aligned(workspace, 16))) return DAT_ERR_ARG;
  hipStream_t st = (hipStream_t)stream;
  GnArgs a{x, dy, gamma, beta, mean, rstd, dx, nullptr, nullptr, (float*)workspace, B, H * W, C, groups, C / groups, 0.0f};
  if (B > 0) {
    const dim3 grid((unsigned)B * groups);
    if (dtype == DAT_BF16) { using T = bf16_t; DAT_GN_LAUNCH(gn_backward_kernel, act); }
    else { using T = float; DAT_GN_LAUNCH(gn_backward_kernel, act); }
    DAT_LAUNCH_CHECK();
  }
  if (dgamma) {
    hipLaunchKernelGGL(gn_param_kernel, dim3((C + kT - 1) / kT), dim3(kT), 0, st, (const float*)workspace, B, C, dgamma, dbeta);
    DAT_LAUNCH_CHECK();
  }
  return DAT_OK;
}
