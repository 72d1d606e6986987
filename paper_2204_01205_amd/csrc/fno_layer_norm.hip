// Layer norm with an activation, forward and adjoint: statistics of every point over its channels, fields [B][C][P] (channels
// first) or [B][P][C] (channels last) in float or bf16.
//
// Plain kernels: a thread has a point and goes over its channels once for the mean, once for the variance and once for the
// result; the adjoint keeps mean and rstd of every point, and a block adds up one channel's sums over all points.
#include "fno_norm_device.h"

namespace fno {

namespace {

struct LayerArgs {
  int B, C;
  long long P, sc, sp;      // strides of a channel and of a point
  float eps;
};
__device__ __forceinline__ long long first_of(const LayerArgs& a, long long q) { return q / a.P * a.C * a.P + q % a.P * a.sp; }

template <class T>
__device__ __forceinline__ double2 stat_of(const LayerArgs& a, const T* x) {
  double s = 0.0, q = 0.0;
  for (int c = 0; c < a.C; ++c) s += load1(x + c * a.sc);
  const double mean = s / a.C;
  for (int c = 0; c < a.C; ++c) {
    const double d = load1(x + c * a.sc) - mean;
    q = fma(d, d, q);
  }
  return make_double2(mean, 1.0 / sqrt(q / a.C + a.eps));
}

template <class T, int ACT>
__global__ __launch_bounds__(kThreads) void layer_fwd_kernel(LayerArgs a, const T* x, const float* gamma, const float* beta, T* y) {
  const long long q = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (q >= a.B * a.P) return;
  const long long at = first_of(a, q);
  const double2 st = stat_of(a, x + at);
  for (int c = 0; c < a.C; ++c) {
    const float z = fmaf((float)((load1(x + at + c * a.sc) - st.x) * st.y), gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
    store1(y + at + c * a.sc, act_f<ACT>(z));
  }
}

template <class T, int ACT>
__global__ __launch_bounds__(kThreads) void layer_bwd_sum_kernel(LayerArgs a, const T* x, const float* gamma, const float* beta,
                                                                 const T* gy, const double2* stat, float* ggamma, float* gbeta, int add) {
  __shared__ double red[2][kThreads / 64];
  const int c = blockIdx.x;
  const float ga = gamma ? gamma[c] : 1.f, be = beta ? beta[c] : 0.f;
  double sg = 0.0, sb = 0.0;
  for (long long q = threadIdx.x; q < a.B * a.P; q += kThreads) {
    const long long at = first_of(a, q) + c * a.sc;
    const float xh = (float)((load1(x + at) - stat[q].x) * stat[q].y);
    const float gz = load1(gy + at) * slope_f<ACT>(kArg<ACT> * fmaf(xh, ga, be));
    sg += gz * xh;
    sb += gz;
  }
  for (int off = 32; off >= 1; off >>= 1) {
    sg += __shfl_xor(sg, off);
    sb += __shfl_xor(sb, off);
  }
  if ((threadIdx.x & 63) == 0) {
    red[0][threadIdx.x >> 6] = sg;
    red[1][threadIdx.x >> 6] = sb;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kThreads / 64; ++w) {
      sg += red[0][w];
      sb += red[1][w];
    }
    if (ggamma) ggamma[c] = (add ? ggamma[c] : 0.f) + (float)sg;
    if (gbeta) gbeta[c] = (add ? gbeta[c] : 0.f) + (float)sb;
  }
}

template <class T>
__global__ __launch_bounds__(kThreads) void layer_stat_kernel(LayerArgs a, const T* x, double2* stat) {
  const long long q = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (q < a.B * a.P) stat[q] = stat_of(a, x + first_of(a, q));
}

template <class T, int ACT>
__global__ __launch_bounds__(kThreads) void layer_bwd_kernel(LayerArgs a, const T* x, const float* gamma, const float* beta, const T* gy,
                                                             const double2* stat, T* gx) {
  const long long q = (long long)blockIdx.x * kThreads + threadIdx.x;
  if (q >= a.B * a.P) return;
  const long long at = first_of(a, q);
  const double2 st = stat[q];
  double t1 = 0.0, t2 = 0.0;
  auto h_of = [&](int c, float& xh) {
    const float ga = gamma ? gamma[c] : 1.f;
    xh = (float)((load1(x + at + c * a.sc) - st.x) * st.y);
    return ga * load1(gy + at + c * a.sc) * slope_f<ACT>(kArg<ACT> * fmaf(xh, ga, beta ? beta[c] : 0.f));
  };
  for (int c = 0; c < a.C; ++c) {
    float xh;
    const float h = h_of(c, xh);
    t1 += h;
    t2 += h * xh;
  }
  const float s1 = (float)(t1 / a.C), s2 = (float)(t2 / a.C);
  for (int c = 0; c < a.C; ++c) {
    float xh;
    const float h = h_of(c, xh);
    store1(gx + at + c * a.sc, (float)st.y * (h - s1 - xh * s2));
  }
}

__global__ void layer_zero_kernel(int C, float* ggamma, float* gbeta) {
  const int c = blockIdx.x * kThreads + threadIdx.x;
  if (c < C && ggamma) ggamma[c] = 0.f;
  if (c < C && gbeta) gbeta[c] = 0.f;
}

template <class F>
void with_kind(const LayerShape& n, F&& f) {
  auto act = [&](auto t) {
    if (n.act == 0) f(t, std::integral_constant<int, 0>());
    else if (n.act == 1) f(t, std::integral_constant<int, 1>());
    else f(t, std::integral_constant<int, 2>());
  };
  if (n.bf16) act(u16());
  else act(float());
}
LayerArgs args_of(const LayerShape& n) {
  return LayerArgs{n.B, n.C, (long long)n.P, n.last ? 1ll : (long long)n.P, n.last ? (long long)n.C : 1ll, (float)n.eps};
}

}  // namespace

size_t layer_norm_workspace_bytes(const LayerShape& n) { return (size_t)(n.B * n.P + 1) * sizeof(double2); }

hipError_t launch_layer_norm_fwd(const LayerShape& n, const void* x, const float* gamma, const float* beta, void* y, hipStream_t s) {
  const dim3 grid((unsigned)((n.B * n.P + kThreads - 1) / kThreads));
  with_kind(n, [&](auto t, auto act) {
    using T = decltype(t);
    hipLaunchKernelGGL((layer_fwd_kernel<T, decltype(act)::value>), grid, dim3(kThreads), 0, s, args_of(n), static_cast<const T*>(x),
                       gamma, beta, static_cast<T*>(y));
  });
  return hipGetLastError();
}

hipError_t launch_layer_norm_bwd(const LayerShape& n, const void* x, const float* gamma, const float* beta, const void* gy,
                                 void* gx, float* ggamma, float* gbeta, int accumulate, void* ws, hipStream_t s) {
  if (n.P == 0) {
    if (!accumulate) hipLaunchKernelGGL(layer_zero_kernel, dim3((n.C + kThreads - 1) / kThreads), dim3(kThreads), 0, s, n.C, ggamma, gbeta);
    return hipGetLastError();
  }
  const dim3 grid((unsigned)((n.B * n.P + kThreads - 1) / kThreads));
  double2* stat = static_cast<double2*>(ws);
  hipError_t e = hipSuccess;
  with_kind(n, [&](auto t, auto act) {
    using T = decltype(t);
    constexpr int A = decltype(act)::value;
    const LayerArgs a = args_of(n);
    const T *xt = static_cast<const T*>(x), *gt = static_cast<const T*>(gy);
    hipLaunchKernelGGL(layer_stat_kernel<T>, grid, dim3(kThreads), 0, s, a, xt, stat);
    if ((e = hipGetLastError()) != hipSuccess) return;
    if (ggamma || gbeta)
      hipLaunchKernelGGL((layer_bwd_sum_kernel<T, A>), dim3(n.C), dim3(kThreads), 0, s, a, xt, gamma, beta, gt, stat, ggamma, gbeta, accumulate);
    if ((e = hipGetLastError()) != hipSuccess) return;
    if (gx) hipLaunchKernelGGL((layer_bwd_kernel<T, A>), grid, dim3(kThreads), 0, s, a, xt, gamma, beta, gt, stat, static_cast<T*>(gx));
    e = hipGetLastError();
  });
  return e;
}

}  // namespace fno
