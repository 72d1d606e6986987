// Group norm with an activation, forward and adjoint, over fields [B][C][P] or [B][P][C] in float or bf16.
#include "fno_device.h"

namespace fno {

namespace {

typedef unsigned short u16;

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const u16* p) { return bf16_low(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(u16* p, float v) { *p = (u16)bf16_pair(v, 0.f); }

template <int ACT>
__device__ __forceinline__ float act_f(float z) {
  if constexpr (ACT == 1) return gelu_fast_f(z);
  if constexpr (ACT == 2) return z / (1.0f + expf(-z));
  return z;
}
template <int ACT>
__device__ __forceinline__ float slope_f(float z) {
  if constexpr (ACT == 1) {
    float v, g;
    gelu_and_grad_f(z, v, g);
    return g;
  }
  if constexpr (ACT == 2) {
    const float s = 1.0f / (1.0f + expf(-z));
    return s * fmaf(z, 1.0f - s, 1.0f);
  }
  return 1.0f;
}

struct NormArgs {
  int C, G, D;          // D = C / G
  long long P;
  int last;
  double inv_n, eps;    // inv_n = 1 / (D P)
};

// place of element q of group g (D P elements, channel outermost) of batch entry b, and its channel
__device__ __forceinline__ long long norm_at(const NormArgs& a, int b, int g, long long q, int& c) {
  c = g * a.D + (int)(q / a.P);
  const long long p = q % a.P;
  return a.last ? ((long long)b * a.P + p) * a.C + c : ((long long)b * a.C + c) * a.P + p;
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < kThreads / 64; ++w) s += red[w];
  return s;
}

// One block per (b, g): mean and variance in double, the variance about the mean.
template <class T>
__global__ __launch_bounds__(kThreads) void norm_stats_kernel(NormArgs a, const T* x, float* mean, float* rstd, double* stat) {
  __shared__ double red[kThreads / 64];
  const int b = blockIdx.x / a.G, g = blockIdx.x % a.G;
  const long long n = a.P * a.D;
  int c;
  double s = 0.0, q = 0.0;
  for (long long i = threadIdx.x; i < n; i += kThreads) s += (double)load1(x + norm_at(a, b, g, i, c));
  const double mu = block_sum(s, red) * a.inv_n;
  for (long long i = threadIdx.x; i < n; i += kThreads) {
    const double d = (double)load1(x + norm_at(a, b, g, i, c)) - mu;
    q += d * d;
  }
  const double rs = 1.0 / sqrt(block_sum(q, red) * a.inv_n + a.eps);
  if (threadIdx.x == 0) {
    if (mean != nullptr) mean[blockIdx.x] = (float)mu;
    if (rstd != nullptr) rstd[blockIdx.x] = (float)rs;
    stat[2 * blockIdx.x] = mu;
    stat[2 * blockIdx.x + 1] = rs;
  }
}

template <class T, int ACT>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs a, const T* x, const float* gamma, const float* beta,
                                                              const double* stat, T* y) {
  const int b = blockIdx.y / a.G, g = blockIdx.y % a.G;
  const double mu = stat[2 * blockIdx.y], rs = stat[2 * blockIdx.y + 1];
  const float hi = (float)mu, lo = (float)(mu - (double)hi);
  const long long n = a.P * a.D;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) {
    int c;
    const long long at = norm_at(a, b, g, i, c);
    const float xh = ((load1(x + at) - hi) - lo) * (float)rs;
    store1(y + at, act_f<ACT>(fmaf(xh, gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f)));
  }
}

// One block per (b, c): S1 = sum gz, S2 = sum gz xh.
template <class T, int ACT>
__global__ __launch_bounds__(kThreads) void norm_sums_kernel(NormArgs a, const T* x, const T* gy, const float* gamma,
                                                             const float* beta, const float* mean, const float* rstd, double* sums) {
  __shared__ double red[kThreads / 64];
  const int b = blockIdx.x / a.C, c = blockIdx.x % a.C, g = c / a.D;
  const float mu = mean[b * a.G + g], rs = rstd[b * a.G + g], ga = gamma ? gamma[c] : 1.f, be = beta ? beta[c] : 0.f;
  double s1 = 0.0, s2 = 0.0;
  for (long long p = threadIdx.x; p < a.P; p += kThreads) {
    int cc;
    const long long at = norm_at(a, b, g, (long long)(c % a.D) * a.P + p, cc);
    const float xh = (load1(x + at) - mu) * rs;
    const float gz = load1(gy + at) * slope_f<ACT>(fmaf(xh, ga, be));
    s1 += gz;
    s2 += (double)gz * xh;
  }
  s1 = block_sum(s1, red);
  s2 = block_sum(s2, red);
  if (threadIdx.x == 0) { sums[2 * blockIdx.x] = s1; sums[2 * blockIdx.x + 1] = s2; }
}

__global__ __launch_bounds__(kThreads) void norm_param_kernel(NormArgs a, int B, const double* sums, float* ggamma, float* gbeta,
                                                              int accumulate) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c >= a.C) return;
  double s1 = 0.0, s2 = 0.0;
  for (int b = 0; b < B; ++b) { s1 += sums[2 * ((long long)b * a.C + c)]; s2 += sums[2 * ((long long)b * a.C + c) + 1]; }
  if (gbeta != nullptr) gbeta[c] = (float)(accumulate ? (double)gbeta[c] + s1 : s1);
  if (ggamma != nullptr) ggamma[c] = (float)(accumulate ? (double)ggamma[c] + s2 : s2);
}

template <class T, int ACT>
__global__ __launch_bounds__(kThreads) void norm_gx_kernel(NormArgs a, const T* x, const T* gy, const float* gamma,
                                                           const float* beta, const float* mean, const float* rstd,
                                                           const double* sums, T* gx) {
  const int b = blockIdx.y / a.G, g = blockIdx.y % a.G;
  const float mu = mean[blockIdx.y], rs = rstd[blockIdx.y];
  double s1 = 0.0, s2 = 0.0;
  for (int d = 0; d < a.D; ++d) {
    const int c = g * a.D + d;
    const double ga = gamma ? gamma[c] : 1.f;
    s1 += ga * sums[2 * ((long long)b * a.C + c)];
    s2 += ga * sums[2 * ((long long)b * a.C + c) + 1];
  }
  const float m1 = (float)(s1 * a.inv_n), m2 = (float)(s2 * a.inv_n);
  const long long n = a.P * a.D;
  for (long long i = (long long)blockIdx.x * kThreads + threadIdx.x; i < n; i += (long long)gridDim.x * kThreads) {
    int c;
    const long long at = norm_at(a, b, g, i, c);
    const float ga = gamma ? gamma[c] : 1.f;
    const float xh = (load1(x + at) - mu) * rs;
    const float gz = load1(gy + at) * slope_f<ACT>(fmaf(xh, ga, beta ? beta[c] : 0.f));
    store1(gx + at, rs * (gz * ga - m1 - xh * m2));
  }
}

NormArgs norm_args(const NormShape& n) {
  const int D = n.C / n.G;
  const double count = (double)n.P * D;
  return NormArgs{n.C, n.G, D, (long long)n.P, n.last ? 1 : 0, count > 0 ? 1.0 / count : 0.0, n.eps};
}

unsigned norm_blocks(const NormArgs& a) {
  const long long nb = (a.P * a.D + 4 * kThreads - 1) / (4 * kThreads);
  return (unsigned)(nb < 1 ? 1 : nb > 4096 ? 4096 : nb);
}

template <class T, int ACT>
hipError_t fwd(const NormShape& n, const void* x, const float* gamma, const float* beta, void* y, float* mean, float* rstd,
               void* ws, hipStream_t s) {
  const NormArgs a = norm_args(n);
  double* stat = static_cast<double*>(ws);
  hipLaunchKernelGGL((norm_stats_kernel<T>), dim3(n.B * n.G), dim3(kThreads), 0, s, a, static_cast<const T*>(x), mean, rstd, stat);
  for (int b = 0; b < n.B && n.P > 0; b += 65535 / n.G)
    hipLaunchKernelGGL((norm_apply_kernel<T, ACT>), dim3(norm_blocks(a), (n.B - b < 65535 / n.G ? n.B - b : 65535 / n.G) * n.G),
                       dim3(kThreads), 0, s, a, static_cast<const T*>(x) + (long long)b * n.C * n.P, gamma, beta,
                       stat + 2ll * b * n.G, static_cast<T*>(y) + (long long)b * n.C * n.P);
  return hipGetLastError();
}

template <class T, int ACT>
hipError_t bwd(const NormShape& n, const void* x, const float* gamma, const float* beta, const float* mean, const float* rstd,
               const void* gy, void* gx, float* ggamma, float* gbeta, int accumulate, void* ws, hipStream_t s) {
  const NormArgs a = norm_args(n);
  double* sums = static_cast<double*>(ws);
  hipLaunchKernelGGL((norm_sums_kernel<T, ACT>), dim3((unsigned)(n.B * n.C)), dim3(kThreads), 0, s, a, static_cast<const T*>(x),
                     static_cast<const T*>(gy), gamma, beta, mean, rstd, sums);
  if (ggamma != nullptr || gbeta != nullptr)
    hipLaunchKernelGGL(norm_param_kernel, dim3((n.C + kThreads - 1) / kThreads), dim3(kThreads), 0, s, a, n.B, sums, ggamma, gbeta,
                       accumulate);
  for (int b = 0; b < n.B && n.P > 0 && gx != nullptr; b += 65535 / n.G) {
    const long long at = (long long)b * n.C * n.P;
    hipLaunchKernelGGL((norm_gx_kernel<T, ACT>), dim3(norm_blocks(a), (n.B - b < 65535 / n.G ? n.B - b : 65535 / n.G) * n.G),
                       dim3(kThreads), 0, s, a, static_cast<const T*>(x) + at, static_cast<const T*>(gy) + at, gamma, beta,
                       mean + (long long)b * n.G, rstd + (long long)b * n.G, sums + 2ll * b * n.C, static_cast<T*>(gx) + at);
  }
  return hipGetLastError();
}

#define FNO_NORM_DISPATCH(FN, ...)                                      \
  if (n.bf16) {                                                         \
    if (n.act == 1) return FN<u16, 1>(__VA_ARGS__);                     \
    if (n.act == 2) return FN<u16, 2>(__VA_ARGS__);                     \
    return FN<u16, 0>(__VA_ARGS__);                                     \
  }                                                                     \
  if (n.act == 1) return FN<float, 1>(__VA_ARGS__);                     \
  if (n.act == 2) return FN<float, 2>(__VA_ARGS__);                     \
  return FN<float, 0>(__VA_ARGS__);

}  // namespace

size_t group_norm_workspace_bytes(const NormShape& n) {
  const size_t bytes = (size_t)n.B * n.C * 2 * sizeof(double);
  return (bytes + 255) & ~size_t(255);
}

hipError_t launch_group_norm_fwd(const NormShape& n, const void* x, const float* gamma, const float* beta, void* y,
                                 float* mean, float* rstd, void* ws, hipStream_t s) {
  FNO_NORM_DISPATCH(fwd, n, x, gamma, beta, y, mean, rstd, ws, s)
}

hipError_t launch_group_norm_bwd(const NormShape& n, const void* x, const float* gamma, const float* beta, const float* mean,
                                 const float* rstd, const void* gy, void* gx, float* ggamma, float* gbeta, int accumulate,
                                 void* ws, hipStream_t s) {
  FNO_NORM_DISPATCH(bwd, n, x, gamma, beta, mean, rstd, gy, gx, ggamma, gbeta, accumulate, ws, s)
}

}  // namespace fno
