// One Muon step over a list of matrices: momentum, its Newton-Schulz products, and the weights.
//
// Plain kernel: a block has a matrix, keeps X, its Gram matrix and the polynomial of it in scratch, and a thread an entry of
// each product at a time.
#include "fno_muon.h"

namespace fno {

namespace {

struct MuonArgs {
  float *p, *mom;
  const float *g, *norm;
  long long batch, si, sj, sb;   // strides, in values, of the shorter side, the longer one and of the matrices
  int m, n, iterations, nesterov;
  float mu, keep, move, a, b, c, max_norm;
  double eps;
  float* ws;
};

__device__ __forceinline__ float2 load_value(const float* p, long long at, bool cplx) {
  return cplx ? reinterpret_cast<const float2*>(p)[at] : make_float2(p[at], 0.f);
}
__device__ __forceinline__ void store_value(float* p, long long at, bool cplx, float2 v) {
  if (cplx) reinterpret_cast<float2*>(p)[at] = v;
  else p[at] = v.x;
}

template <bool CPLX>
__global__ __launch_bounds__(kThreads) void muon_plain_kernel(MuonArgs t) {
  __shared__ double red[kThreads / 64];
  float scale = 1.0f;
  if (t.norm != nullptr) {
    const float norm = *t.norm;
    if (!(norm <= 3.402823466e38f)) return;
    if (norm > t.max_norm) scale = t.max_norm / norm;
  }
  const int m = t.m, n = t.n;
  const size_t each = 2 * (size_t)m * n + 2 * (size_t)m * m;
  float2* const x0 = reinterpret_cast<float2*>(t.ws) + blockIdx.x * each;
  float2 *const x1 = x0 + (size_t)m * n, *const A = x1 + (size_t)m * n, *const Q = A + (size_t)m * m;
  for (long long k = blockIdx.x; k < t.batch; k += gridDim.x) {
    double sum = 0.0;
    for (int e = threadIdx.x; e < m * n; e += kThreads) {
      const long long at = k * t.sb + e / n * t.si + e % n * t.sj;
      const float2 g = load_value(t.g, at, CPLX), old = load_value(t.mom, at, CPLX);
      const float gx = g.x * scale, gy = g.y * scale;
      const float2 mo = make_float2(t.mu * old.x + gx, t.mu * old.y + gy);
      store_value(t.mom, at, CPLX, mo);
      const float2 u = t.nesterov ? make_float2(gx + t.mu * mo.x, gy + t.mu * mo.y) : mo;
      x0[e] = u;
      sum += (double)u.x * u.x + (double)u.y * u.y;
    }
    for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = (red[0] + red[1]) + (red[2] + red[3]);
    const double size = sqrt(sum) + t.eps, inv = sum == 0.0 ? 0.0 : 1.0 / size;
    for (int e = threadIdx.x; e < m * n; e += kThreads) x0[e] = make_float2((float)(x0[e].x * inv), (float)(x0[e].y * inv));
    __syncthreads();
    float2 *x = x0, *y = x1;
    for (int it = 0; it < t.iterations; ++it) {
      for (int e = threadIdx.x; e < m * m; e += kThreads) {
        const float2 *r = x + (size_t)(e / m) * n, *q = x + (size_t)(e % m) * n;
        float2 s = make_float2(0.f, 0.f);
        for (int c = 0; c < n; ++c) {
          s.x += r[c].x * q[c].x + r[c].y * q[c].y;
          s.y += r[c].y * q[c].x - r[c].x * q[c].y;
        }
        A[e] = s;
      }
      __syncthreads();
      for (int e = threadIdx.x; e < m * m; e += kThreads) {
        const int i = e / m, j = e % m;
        float2 s = make_float2(0.f, 0.f);
        for (int c = 0; c < m; ++c) {
          const float2 l = A[i * m + c], r = A[c * m + j];
          s.x += l.x * r.x - l.y * r.y;
          s.y += l.x * r.y + l.y * r.x;
        }
        Q[e] = make_float2(t.b * A[e].x + t.c * s.x, t.b * A[e].y + t.c * s.y);
      }
      __syncthreads();
      for (int e = threadIdx.x; e < m * n; e += kThreads) {
        const int i = e / n, j = e % n;
        float2 s = make_float2(0.f, 0.f);
        for (int c = 0; c < m; ++c) {
          const float2 l = Q[i * m + c], r = x[(size_t)c * n + j];
          s.x += l.x * r.x - l.y * r.y;
          s.y += l.x * r.y + l.y * r.x;
        }
        y[e] = make_float2(t.a * x[e].x + s.x, t.a * x[e].y + s.y);
      }
      __syncthreads();
      float2* const z = x;
      x = y;
      y = z;
    }
    for (int e = threadIdx.x; e < m * n; e += kThreads) {
      const long long at = k * t.sb + e / n * t.si + e % n * t.sj;
      const float2 p = load_value(t.p, at, CPLX);
      store_value(t.p, at, CPLX, make_float2(p.x * t.keep - t.move * x[e].x, p.y * t.keep - t.move * x[e].y));
    }
    __syncthreads();
  }
}

constexpr long long kBlocks = 512;
size_t scratch_of(const MuonTensor& t) {
  const size_t m = t.rows < t.cols ? t.rows : t.cols, n = t.rows < t.cols ? t.cols : t.rows;
  return (size_t)(t.batch < kBlocks ? t.batch : kBlocks) * (2 * m * n + 2 * m * m) * sizeof(float2);
}

}  // namespace

size_t muon_workspace_bytes(const MuonTensor* t, int count) {
  size_t most = 0;
  for (int k = 0; k < count; ++k)
    if (!t[k].modes && !muon_is_small(t[k])) most = scratch_of(t[k]) > most ? scratch_of(t[k]) : most;
  return most;
}

hipError_t launch_muon(const MuonTensor* t, int count, const MuonStep& st, void* ws, hipStream_t s) {
  const MuonScalars c{(float)st.momentum, (float)st.a, (float)st.b, (float)st.c, (float)st.max_norm, st.nesterov ? 1 : 0,
                      st.iterations, st.eps, st.norm};
  hipError_t e = launch_muon_modes(t, count, c, st.lr, s);
  if (e != hipSuccess) return e;
  e = launch_muon_small(t, count, c, st.lr, s);
  if (e != hipSuccess) return e;
  for (int k = 0; k < count; ++k) {
    if (t[k].modes || muon_is_small(t[k])) continue;
    const bool tall = t[k].rows > t[k].cols;
    const long long row = t[k].modes ? t[k].cols * t[k].batch : t[k].cols, col = t[k].modes ? t[k].batch : 1;
    const MuonArgs a{t[k].p, t[k].m, t[k].g, st.norm, (long long)t[k].batch, tall ? col : row, tall ? row : col,
                     t[k].modes ? 1ll : (long long)t[k].rows * t[k].cols, tall ? t[k].cols : t[k].rows, tall ? t[k].rows : t[k].cols,
                     st.iterations, st.nesterov ? 1 : 0, (float)st.momentum, (float)(1.0 - st.lr * t[k].decay),
                     (float)(st.lr * t[k].scale), (float)st.a, (float)st.b, (float)st.c, (float)st.max_norm, st.eps,
                     static_cast<float*>(ws)};
    const dim3 grid((unsigned)(t[k].batch < kBlocks ? t[k].batch : kBlocks));
    if (t[k].modes) hipLaunchKernelGGL(muon_plain_kernel<true>, grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL(muon_plain_kernel<false>, grid, dim3(kThreads), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fno
