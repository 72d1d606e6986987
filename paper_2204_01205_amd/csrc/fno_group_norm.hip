// Group norm with an activation, forward and adjoint, over fields [B][C][P] (channels first) or [B][P][C] (channels
// last) in float or bf16.
//
// What the operator moves bounds it: x in and y out (adjoint: x and gy in, gx out), 20 to 40 operations a value.  The
// statistics (adjoint: the sums) of a group need all of it before its first output, so a group that does not fit one
// block's registers is read twice: sums of pieces, a small launch that adds the pieces' sums in a fixed order, and the
// sweep that writes.  The statistics come from d = x - k, k the group's first value: mean = k + E d, var = E d^2 - (E d)^2,
// sums in double, so that values far from zero lose nothing and a constant group has the variance zero.
#include "fno_device.h"

#include <type_traits>

namespace fno {

namespace {

typedef unsigned short u16;
template <class T> constexpr int kVec = 16 / (int)sizeof(T);      // values of a 16-byte access

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const u16* p) { return bf16_low(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(u16* p, float v) { *p = (u16)bf16_pair(v, 0.f); }

// 16 bytes at an aligned address, and the values in them
template <class T> struct pack_of;
template <> struct pack_of<float> { typedef v4f type; };
template <> struct pack_of<u16> { typedef u32x4 type; };
template <class T> using pack = typename pack_of<T>::type;
template <class T>
__device__ __forceinline__ pack<T> load_pack(const T* p) { return *reinterpret_cast<const pack<T>*>(p); }
template <class T>
__device__ __forceinline__ void store_pack(T* p, pack<T> v) { *reinterpret_cast<pack<T>*>(p) = v; }
__device__ __forceinline__ void unpack(v4f q, float (&v)[4]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) v[u] = q[u];
}
__device__ __forceinline__ void unpack(u32x4 q, float (&v)[8]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    v[2 * u] = bf16_low(q[u]);
    v[2 * u + 1] = bf16_high(q[u]);
  }
}
__device__ __forceinline__ v4f repack(const float (&v)[4]) { return v4f{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ u32x4 repack(const float (&v)[8]) {
  return u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
}

// exp(-z) as a power of two; for z below -88 it is infinite and the sigmoid zero, as in the definition
__device__ __forceinline__ float sigmoid_f(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504089f));
}
template <int ACT>
__device__ __forceinline__ float act_f(float z) {
  if constexpr (ACT == 1) return gelu_fast_f(z);
  if constexpr (ACT == 2) return z * sigmoid_f(z);
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
    const float s = sigmoid_f(z);
    return s * fmaf(z, 1.0f - s, 1.0f);
  }
  return 1.0f;
}

struct NormArgs {
  int B, C, G, D;       // D = C / G
  long long P;
  double inv_n, eps;    // inv_n = 1 / (D P)
  // pieces: of a group (forward, channels first), of a row (adjoint, channels first), of a batch entry (channels last)
  int pieces;
  long long per;        // values, or points (channels last), of a piece
};

// What a group's values go through: xh = (x - mean) rstd with the mean in two floats, so that x - hi is exact near it.
struct Stat {
  float hi, lo, rstd, pad;
};
__device__ __forceinline__ Stat stat_of(double k, double sum, double square, const NormArgs& a, float* mean, float* rstd,
                                        long long at) {
  const double off = sum * a.inv_n, mu = k + off;
  double var = square * a.inv_n - off * off;
  if (var < 0.0) var = 0.0;                              // (a NaN stays one)
  const double rs = 1.0 / sqrt(var + a.eps);
  if (mean != nullptr) mean[at] = (float)mu;
  if (rstd != nullptr) rstd[at] = (float)rs;
  Stat s;
  s.hi = (float)mu;
  s.lo = (float)(mu - (double)s.hi);
  s.rstd = (float)rs;
  s.pad = 0.f;
  return s;
}

__device__ __forceinline__ void wave_sum2(double& a, double& b) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) {
    a += __shfl_xor(a, off);
    b += __shfl_xor(b, off);
  }
}
// sums over the block, in every thread; red: two doubles a wave
__device__ __forceinline__ void block_sum2(double& a, double& b, double* red) {
  wave_sum2(a, b);
  const int nw = (blockDim.x + 63) >> 6;
  if ((threadIdx.x & 63) == 0) {
    red[2 * (threadIdx.x >> 6)] = a;
    red[2 * (threadIdx.x >> 6) + 1] = b;
  }
  __syncthreads();
  a = 0.0;
  b = 0.0;
  for (int w = 0; w < nw; ++w) {
    a += red[2 * w];
    b += red[2 * w + 1];
  }
}

// Calls vec(at) for the 16-byte pieces of [begin, end) that start at multiples of their length, U of them at a time in
// vecs(at, step), and one(at) for the values before and behind them.  Places count from a 16-byte aligned base.
template <int V, int U, class FVecs, class FVec, class FOne>
__device__ __forceinline__ void sweep(long long begin, long long end, int tid, int threads, FVecs&& vecs, FVec&& vec, FOne&& one) {
  long long lo = (begin + V - 1) / V * V;
  if (lo > end) lo = end;
  const long long hi = lo + (end - lo) / V * V;
  if (begin + tid < lo) one(begin + tid);
  if (hi + tid < end) one(hi + tid);
  const long long step = (long long)threads * V;
  long long at = lo + (long long)tid * V;
  for (; at + (U - 1) * step < hi; at += U * step) vecs(at, step);
  for (; at < hi; at += step) vec(at);
}

// ------------------------------------------------------------------------------------------
// Channels first.  A group's values lie together: pieces of them whatever the channel for the statistics; a block's
// piece of one row (one channel), or whole short rows wave by wave, where gamma and beta come in.
// ------------------------------------------------------------------------------------------

// part[(bg, piece)] = (sum d, sum d^2)
template <class T>
__global__ __launch_bounds__(kThreads) void norm_sum_kernel(NormArgs a, const T* x, double2* part) {
  constexpr int V = kVec<T>, U = 4;
  __shared__ double red[2 * kThreads / 64];
  const long long bg = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces, n = a.P * a.D;
  const long long begin = bg * n + j * a.per, end = j * a.per + a.per < n ? begin + a.per : (bg + 1) * n;
  const float first = a.P > 0 ? load1(x + bg * n) : 0.f;
  double s = 0.0, q = 0.0;
  auto add1 = [&](float v) {
    const double d = v - first;
    s += d;
    q = fma(d, d, q);
  };
  auto add = [&](pack<T> k) {
    float v[V];
    unpack(k, v);
#pragma unroll
    for (int u = 0; u < V; ++u) add1(v[u]);
  };
  sweep<V, U>(begin, end, threadIdx.x, kThreads,
              [&](long long at, long long step) {
                pack<T> k[U];
#pragma unroll
                for (int u = 0; u < U; ++u) k[u] = load_pack(x + at + u * step);
#pragma unroll
                for (int u = 0; u < U; ++u) add(k[u]);
              },
              [&](long long at) { add(load_pack(x + at)); },
              [&](long long at) { add1(load1(x + at)); });
  block_sum2(s, q, red);
  if (threadIdx.x == 0) part[blockIdx.x] = make_double2(s, q);
}

// Adds the pieces of every (b, g): part[bg][piece] -> stat[bg], mean, rstd.
template <class T, bool LAST>
__global__ __launch_bounds__(kThreads) void norm_stat_kernel(NormArgs a, const T* x, const double2* part, Stat* stat, float* mean,
                                                             float* rstd) {
  __shared__ double red[2 * kThreads / 64];
  double s = 0.0, q = 0.0;
  for (int j = threadIdx.x; j < a.pieces; j += kThreads) {
    const double2 p = part[(long long)blockIdx.x * a.pieces + j];
    s += p.x;
    q += p.y;
  }
  block_sum2(s, q, red);
  if (threadIdx.x != 0) return;
  const long long b = blockIdx.x / a.G, c = (long long)(blockIdx.x % a.G) * a.D;
  const double first = a.P > 0 ? load1(x + (LAST ? b * a.P * a.C + c : (b * a.C + c) * a.P)) : 0.f;
  stat[blockIdx.x] = stat_of(first, s, q, a, mean, rstd, blockIdx.x);
}

// What one channel's values go through
struct Affine {
  float hi, scale, shift;      // act((x - hi) scale + shift)
};
__device__ __forceinline__ Affine affine_of(const Stat& s, float gamma, float beta) {
  Affine f;
  f.hi = s.hi;
  f.scale = s.rstd * gamma;
  f.shift = fmaf(-s.lo, f.scale, beta);
  return f;
}
template <int ACT>
__device__ __forceinline__ float normed(const Affine& f, float x) { return act_f<ACT>(fmaf(x - f.hi, f.scale, f.shift)); }

template <class T, int ACT>
__device__ __forceinline__ void apply_range(const Affine& f, const T* x, T* y, long long begin, long long end, int tid, int threads) {
  constexpr int V = kVec<T>, U = 4;
  auto put = [&](long long at, pack<T> k) {
    float v[V];
    unpack(k, v);
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = normed<ACT>(f, v[u]);
    store_pack(y + at, repack(v));
  };
  sweep<V, U>(begin, end, tid, threads,
              [&](long long at, long long step) {
                pack<T> k[U];
#pragma unroll
                for (int u = 0; u < U; ++u) k[u] = load_pack(x + at + u * step);
#pragma unroll
                for (int u = 0; u < U; ++u) put(at + u * step, k[u]);
              },
              [&](long long at) { put(at, load_pack(x + at)); },
              [&](long long at) { store1(y + at, normed<ACT>(f, load1(x + at))); });
}

// A piece of a row per block; short: a row per wave.
template <class T, int ACT, bool SHORT>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs a, const T* x, const float* gamma, const float* beta,
                                                              const Stat* stat, T* y) {
  const long long row = SHORT ? (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6) : blockIdx.x / a.pieces;
  if (SHORT && row >= (long long)a.B * a.C) return;
  const int c = (int)(row % a.C);
  const Affine f = affine_of(stat[row / a.D], gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
  const long long j = SHORT ? 0 : blockIdx.x % a.pieces;
  const long long begin = row * a.P + j * a.per, end = SHORT || (j + 1) * a.per >= a.P ? (row + 1) * a.P : begin + a.per;
  if (SHORT) apply_range<T, ACT>(f, x, y, begin, end, threadIdx.x & 63, 64);
  else apply_range<T, ACT>(f, x, y, begin, end, threadIdx.x, kThreads);
}

// The adjoint's terms of one value
struct Slope {
  float mean, rstd, gamma, beta;
};
template <int ACT>
__device__ __forceinline__ void terms(const Slope& k, float x, float gy, float& xh, float& gz) {
  xh = (x - k.mean) * k.rstd;
  gz = ACT == 0 ? gy : gy * slope_f<ACT>(fmaf(xh, k.gamma, k.beta));
}

// part[(row, piece)] = (sum gz, sum gz xh)
template <class T, int ACT, bool SHORT>
__global__ __launch_bounds__(kThreads) void norm_grad_sum_kernel(NormArgs a, const T* x, const T* gy, const float* gamma,
                                                                 const float* beta, const float* mean, const float* rstd,
                                                                 double2* part) {
  constexpr int V = kVec<T>, U = 2;
  __shared__ double red[2 * kThreads / 64];
  const long long row = SHORT ? (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6) : blockIdx.x / a.pieces;
  if (SHORT && row >= (long long)a.B * a.C) return;
  const int c = (int)(row % a.C);
  const long long bg = row / a.D;
  const Slope k{mean[bg], rstd[bg], gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f};
  const long long j = SHORT ? 0 : blockIdx.x % a.pieces;
  const long long begin = row * a.P + j * a.per, end = SHORT || (j + 1) * a.per >= a.P ? (row + 1) * a.P : begin + a.per;
  double s1 = 0.0, s2 = 0.0;
  auto add = [&](pack<T> px, pack<T> pg) {
    float v[V], g[V], t1 = 0.f, t2 = 0.f;
    unpack(px, v);
    unpack(pg, g);
#pragma unroll
    for (int u = 0; u < V; ++u) {
      float xh, gz;
      terms<ACT>(k, v[u], g[u], xh, gz);
      t1 += gz;
      t2 = fmaf(gz, xh, t2);
    }
    s1 += t1;                                            // 4 or 8 terms in float, then doubles
    s2 += t2;
  };
  sweep<V, U>(begin, end, SHORT ? threadIdx.x & 63 : threadIdx.x, SHORT ? 64 : kThreads,
              [&](long long at, long long step) {
                pack<T> px[U], pg[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                  px[u] = load_pack(x + at + u * step);
                  pg[u] = load_pack(gy + at + u * step);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) add(px[u], pg[u]);
              },
              [&](long long at) { add(load_pack(x + at), load_pack(gy + at)); },
              [&](long long at) {
                float xh, gz;
                terms<ACT>(k, load1(x + at), load1(gy + at), xh, gz);
                s1 += gz;
                s2 = fma((double)gz, (double)xh, s2);
              });
  if (SHORT) {
    wave_sum2(s1, s2);
    if ((threadIdx.x & 63) == 0) part[row] = make_double2(s1, s2);
  } else {
    block_sum2(s1, s2, red);
    if (threadIdx.x == 0) part[blockIdx.x] = make_double2(s1, s2);
  }
}

// Blocks 0 .. B G - 1: m[bg] = the group's means of gamma gz and gamma gz xh.  The blocks behind: the parameters'
// gradients, a channel a wave.  part[(b, c)][piece].
__global__ __launch_bounds__(kThreads) void norm_grad_fold_kernel(NormArgs a, const double2* part, const float* gamma, float2* m,
                                                                  float* ggamma, float* gbeta, int accumulate) {
  __shared__ double red[2 * kThreads / 64];
  const long long groups = (long long)a.B * a.G;
  double s1 = 0.0, s2 = 0.0;
  if (blockIdx.x < groups) {
    const long long count = (long long)a.D * a.pieces, at = blockIdx.x * count;
    const int c0 = (int)(blockIdx.x % a.G) * a.D;
    for (long long j = threadIdx.x; j < count; j += kThreads) {
      const double2 p = part[at + j];
      const double ga = gamma ? gamma[c0 + (int)(j / a.pieces)] : 1.f;
      s1 = fma(ga, p.x, s1);
      s2 = fma(ga, p.y, s2);
    }
    block_sum2(s1, s2, red);
    if (threadIdx.x == 0) m[blockIdx.x] = make_float2((float)(s1 * a.inv_n), (float)(s2 * a.inv_n));
    return;
  }
  const long long c = (blockIdx.x - groups) * (kThreads / 64) + (threadIdx.x >> 6);
  if (c >= a.C) return;
  const long long count = (long long)a.B * a.pieces;
  for (long long j = threadIdx.x & 63; j < count; j += 64) {
    const double2 p = part[(j / a.pieces * a.C + c) * a.pieces + j % a.pieces];
    s1 += p.x;
    s2 += p.y;
  }
  wave_sum2(s1, s2);
  if ((threadIdx.x & 63) == 0) {
    if (gbeta != nullptr) gbeta[c] = (float)(accumulate ? (double)gbeta[c] + s1 : s1);
    if (ggamma != nullptr) ggamma[c] = (float)(accumulate ? (double)ggamma[c] + s2 : s2);
  }
}

template <int ACT>
__device__ __forceinline__ float grad_of(const Slope& k, float2 m, float x, float gy) {
  float xh, gz;
  terms<ACT>(k, x, gy, xh, gz);
  return k.rstd * (fmaf(gz, k.gamma, -m.x) - xh * m.y);
}

template <class T, int ACT, bool SHORT>
__global__ __launch_bounds__(kThreads) void norm_grad_apply_kernel(NormArgs a, const T* x, const T* gy, const float* gamma,
                                                                   const float* beta, const float* mean, const float* rstd,
                                                                   const float2* m, T* gx) {
  constexpr int V = kVec<T>, U = 2;
  const long long row = SHORT ? (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6) : blockIdx.x / a.pieces;
  if (SHORT && row >= (long long)a.B * a.C) return;
  const int c = (int)(row % a.C);
  const long long bg = row / a.D;
  const Slope k{mean[bg], rstd[bg], gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f};
  const float2 mm = m[bg];
  const long long j = SHORT ? 0 : blockIdx.x % a.pieces;
  const long long begin = row * a.P + j * a.per, end = SHORT || (j + 1) * a.per >= a.P ? (row + 1) * a.P : begin + a.per;
  auto put = [&](long long at, pack<T> px, pack<T> pg) {
    float v[V], g[V];
    unpack(px, v);
    unpack(pg, g);
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = grad_of<ACT>(k, mm, v[u], g[u]);
    store_pack(gx + at, repack(v));
  };
  sweep<V, U>(begin, end, SHORT ? threadIdx.x & 63 : threadIdx.x, SHORT ? 64 : kThreads,
              [&](long long at, long long step) {
                pack<T> px[U], pg[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                  px[u] = load_pack(x + at + u * step);
                  pg[u] = load_pack(gy + at + u * step);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) put(at + u * step, px[u], pg[u]);
              },
              [&](long long at) { put(at, load_pack(x + at), load_pack(gy + at)); },
              [&](long long at) { store1(gx + at, grad_of<ACT>(k, mm, load1(x + at), load1(gy + at))); });
}

// ------------------------------------------------------------------------------------------
// Channels last.  The points of a batch entry lie one behind the other, C values each.  `active` threads take 16 bytes each,
// one behind the other; active x V is a multiple of C, so that a thread meets the same V channels in every step: their
// factors and sums stay in its registers, and no access knows of channels.  Batch entries whose start is not 16-byte
// aligned are read and written in 16-byte accesses at their values' own alignment.
// ------------------------------------------------------------------------------------------

template <class T>
__device__ __forceinline__ pack<T> load_any(const T* p) {
  typedef pack<T> loose __attribute__((aligned(sizeof(T))));
  return *reinterpret_cast<const loose*>(p);
}
template <class T>
__device__ __forceinline__ void store_any(T* p, pack<T> v) {
  typedef pack<T> loose __attribute__((aligned(sizeof(T))));
  *reinterpret_cast<loose*>(p) = v;
}

// Calls vecs(at, step), vec(at) and one(at, u) (u: which of the thread's channels) over the values [begin, end) of whole
// points; the last 16 bytes may be cut.
template <int V, int U, class FVecs, class FVec, class FOne>
__device__ __forceinline__ void sweep_last(long long begin, long long end, int active, FVecs&& vecs, FVec&& vec, FOne&& one) {
  if ((int)threadIdx.x >= active) return;
  const long long step = (long long)active * V;
  long long at = begin + (long long)threadIdx.x * V;
  for (; at + (U - 1) * step + V <= end; at += U * step) vecs(at, step);
  for (; at + V <= end; at += step) vec(at);
  for (int u = 0; u < V; ++u)
    if (at + u < end) one(at + u, u);
}

// lds[e], e < rows * C: sums over the rows, and then over the channels of every group where D > 1, left in lds[g * D].
__device__ __forceinline__ void tree(double* lds, int rows, int width) {
  while (rows > 1) {
    const int h = (rows + 1) >> 1;
    __syncthreads();
    for (int i = threadIdx.x; i < (rows - h) * width; i += blockDim.x) lds[i] += lds[i + h * width];
    rows = h;
  }
  __syncthreads();
}
__device__ __forceinline__ void tree_groups(double* lds, int G, int D) {
  int n = D;
  while (n > 1) {
    const int h = (n + 1) >> 1;
    for (int i = threadIdx.x; i < G * (n - h); i += blockDim.x) {
      const int g = i / (n - h), d = i % (n - h);
      lds[g * D + d] += lds[g * D + d + h];
    }
    n = h;
    __syncthreads();
  }
}

// part[(b, g)][piece] = (sum d, sum d^2)
template <class T>
__global__ __launch_bounds__(1024) void norm_last_sum_kernel(NormArgs a, int active, const T* x, double* part) {
  constexpr int V = kVec<T>, U = 4;
  extern __shared__ double lds[];
  const int b = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  const long long p0 = (long long)j * a.per, p1 = p0 + a.per < a.P ? p0 + a.per : a.P;
  const long long base = (long long)b * a.P * a.C;
  double s[V], q[V];
  float first[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    s[u] = q[u] = 0.0;
    first[u] = a.P > 0 ? load1(x + base + ((int)threadIdx.x * V + u) % a.C / a.D * a.D) : 0.f;
  }
  auto add1 = [&](int u, float v) {
    const double d = v - first[u];
    s[u] += d;
    q[u] = fma(d, d, q[u]);
  };
  auto add = [&](pack<T> k) {
    float v[V];
    unpack(k, v);
#pragma unroll
    for (int u = 0; u < V; ++u) add1(u, v[u]);
  };
  sweep_last<V, U>(base + p0 * a.C, base + p1 * a.C, active,
                   [&](long long at, long long step) {
                     pack<T> k[U];
#pragma unroll
                     for (int u = 0; u < U; ++u) k[u] = load_any(x + at + u * step);
#pragma unroll
                     for (int u = 0; u < U; ++u) add(k[u]);
                   },
                   [&](long long at) { add(load_any(x + at)); },
                   [&](long long at, int u) {
                     const float v = load1(x + at);
#pragma unroll
                     for (int w = 0; w < V; ++w)
                       if (w == u) add1(w, v);
                   });
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if ((int)threadIdx.x < active) {
#pragma unroll
      for (int u = 0; u < V; ++u) lds[threadIdx.x * V + u] = half ? q[u] : s[u];
    }
    tree(lds, active * V / a.C, a.C);
    tree_groups(lds, a.G, a.D);
    for (int g = threadIdx.x; g < a.G; g += blockDim.x)
      part[2 * (((long long)b * a.G + g) * a.pieces + j) + half] = lds[g * a.D];
    __syncthreads();
  }
}

template <class T, int ACT>
__global__ __launch_bounds__(1024) void norm_last_apply_kernel(NormArgs a, int active, const T* x, const float* gamma,
                                                               const float* beta, const Stat* stat, T* y) {
  constexpr int V = kVec<T>, U = 4;
  const int b = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  const long long p0 = (long long)j * a.per, p1 = p0 + a.per < a.P ? p0 + a.per : a.P;
  const long long base = (long long)b * a.P * a.C;
  Affine f[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int c = ((int)threadIdx.x * V + u) % a.C;
    f[u] = affine_of(stat[(long long)b * a.G + c / a.D], gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
  }
  auto put = [&](long long at, pack<T> k) {
    float v[V];
    unpack(k, v);
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = normed<ACT>(f[u], v[u]);
    store_any(y + at, repack(v));
  };
  sweep_last<V, U>(base + p0 * a.C, base + p1 * a.C, active,
                   [&](long long at, long long step) {
                     pack<T> k[U];
#pragma unroll
                     for (int u = 0; u < U; ++u) k[u] = load_any(x + at + u * step);
#pragma unroll
                     for (int u = 0; u < U; ++u) put(at + u * step, k[u]);
                   },
                   [&](long long at) { put(at, load_any(x + at)); },
                   [&](long long at, int u) {
                     Affine g = f[0];
#pragma unroll
                     for (int w = 1; w < V; ++w)
                       if (w == u) g = f[w];
                     store1(y + at, normed<ACT>(g, load1(x + at)));
                   });
}

// the slopes of a thread's channels
template <int V>
__device__ __forceinline__ void slopes_of(const NormArgs& a, int b, const float* gamma, const float* beta, const float* mean,
                                          const float* rstd, Slope (&k)[V]) {
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int c = ((int)threadIdx.x * V + u) % a.C;
    const long long bg = (long long)b * a.G + c / a.D;
    k[u] = Slope{mean[bg], rstd[bg], gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f};
  }
}

// part[(b, c)][piece] = (sum gz, sum gz xh)
template <class T, int ACT>
__global__ __launch_bounds__(1024) void norm_last_grad_sum_kernel(NormArgs a, int active, const T* x, const T* gy,
                                                                  const float* gamma, const float* beta, const float* mean,
                                                                  const float* rstd, double* part) {
  constexpr int V = kVec<T>, U = 2;
  extern __shared__ double lds[];
  const int b = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  const long long p0 = (long long)j * a.per, p1 = p0 + a.per < a.P ? p0 + a.per : a.P;
  const long long base = (long long)b * a.P * a.C;
  Slope k[V];
  slopes_of<V>(a, b, gamma, beta, mean, rstd, k);
  double s1[V], s2[V];
#pragma unroll
  for (int u = 0; u < V; ++u) s1[u] = s2[u] = 0.0;
  auto add1 = [&](int u, float v, float g) {
    float xh, gz;
    terms<ACT>(k[u], v, g, xh, gz);
    s1[u] += gz;
    s2[u] = fma((double)gz, (double)xh, s2[u]);
  };
  auto add = [&](pack<T> px, pack<T> pg) {
    float v[V], g[V];
    unpack(px, v);
    unpack(pg, g);
#pragma unroll
    for (int u = 0; u < V; ++u) add1(u, v[u], g[u]);
  };
  sweep_last<V, U>(base + p0 * a.C, base + p1 * a.C, active,
                   [&](long long at, long long step) {
                     pack<T> px[U], pg[U];
#pragma unroll
                     for (int u = 0; u < U; ++u) {
                       px[u] = load_any(x + at + u * step);
                       pg[u] = load_any(gy + at + u * step);
                     }
#pragma unroll
                     for (int u = 0; u < U; ++u) add(px[u], pg[u]);
                   },
                   [&](long long at) { add(load_any(x + at), load_any(gy + at)); },
                   [&](long long at, int u) {
                     const float v = load1(x + at), g = load1(gy + at);
#pragma unroll
                     for (int w = 0; w < V; ++w)
                       if (w == u) add1(w, v, g);
                   });
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    if ((int)threadIdx.x < active) {
#pragma unroll
      for (int u = 0; u < V; ++u) lds[threadIdx.x * V + u] = half ? s2[u] : s1[u];
    }
    tree(lds, active * V / a.C, a.C);
    for (int c = threadIdx.x; c < a.C; c += blockDim.x) part[2 * (((long long)b * a.C + c) * a.pieces + j) + half] = lds[c];
    __syncthreads();
  }
}

template <class T, int ACT>
__global__ __launch_bounds__(1024) void norm_last_grad_apply_kernel(NormArgs a, int active, const T* x, const T* gy,
                                                                    const float* gamma, const float* beta, const float* mean,
                                                                    const float* rstd, const float2* m, T* gx) {
  constexpr int V = kVec<T>, U = 2;
  const int b = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  const long long p0 = (long long)j * a.per, p1 = p0 + a.per < a.P ? p0 + a.per : a.P;
  const long long base = (long long)b * a.P * a.C;
  Slope k[V];
  slopes_of<V>(a, b, gamma, beta, mean, rstd, k);
  float2 mm[V];
#pragma unroll
  for (int u = 0; u < V; ++u) mm[u] = m[(long long)b * a.G + (((int)threadIdx.x * V + u) % a.C) / a.D];
  auto put = [&](long long at, pack<T> px, pack<T> pg) {
    float v[V], g[V];
    unpack(px, v);
    unpack(pg, g);
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = grad_of<ACT>(k[u], mm[u], v[u], g[u]);
    store_any(gx + at, repack(v));
  };
  sweep_last<V, U>(base + p0 * a.C, base + p1 * a.C, active,
                   [&](long long at, long long step) {
                     pack<T> px[U], pg[U];
#pragma unroll
                     for (int u = 0; u < U; ++u) {
                       px[u] = load_any(x + at + u * step);
                       pg[u] = load_any(gy + at + u * step);
                     }
#pragma unroll
                     for (int u = 0; u < U; ++u) put(at + u * step, px[u], pg[u]);
                   },
                   [&](long long at) { put(at, load_any(x + at), load_any(gy + at)); },
                   [&](long long at, int u) {
                     const float v = load1(x + at), g = load1(gy + at);
#pragma unroll
                     for (int w = 0; w < V; ++w)
                       if (w == u) store1(gx + at, grad_of<ACT>(k[w], mm[w], v, g));
                   });
}

// ------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------
constexpr long long kNormBlocks = 4096;       // blocks that a sweep is cut into: 16 a CU
constexpr long long kLeastPiece = 8192;       // values
constexpr long long kShortRow = 2048;         // rows below this go wave by wave

NormArgs norm_args(const NormShape& n) {
  const int D = n.C / n.G;
  const double count = (double)n.P * D;
  return NormArgs{n.B, n.C, n.G, D, (long long)n.P, count > 0 ? 1.0 / count : 0.0, n.eps, 1, 0};
}

// Cuts each of `ranges` ranges of `length` into pieces of a multiple of `unit`.
void cut(NormArgs& a, long long ranges, long long length, long long unit, long long least) {
  long long pieces = (kNormBlocks + ranges - 1) / ranges;
  const long long most = length / least;
  if (pieces > most) pieces = most;
  if (pieces < 1) pieces = 1;
  long long per = (length + pieces - 1) / pieces;
  per = (per + unit - 1) / unit * unit;
  if (per < unit) per = unit;
  pieces = (length + per - 1) / per;
  a.pieces = (int)(pieces < 1 ? 1 : pieces);
  a.per = per;
}
NormArgs cut_groups(const NormShape& n) {              // channels first, statistics
  NormArgs a = norm_args(n);
  cut(a, (long long)n.B * n.G, a.P * a.D, 8, kLeastPiece);
  return a;
}
NormArgs cut_rows(const NormShape& n) {                // channels first, where channels count
  NormArgs a = norm_args(n);
  if (n.P < kShortRow) { a.pieces = 1; a.per = n.P; }
  else cut(a, (long long)n.B * n.C, n.P, 8, kLeastPiece);
  return a;
}
NormArgs cut_points(const NormShape& n) {              // channels last: pieces of at least 64 points, whose sums (16 bytes a
  NormArgs a = norm_args(n);                           // channel) are then little beside them
  const long long least = kLeastPiece / n.C > 64 ? kLeastPiece / n.C : 64;
  cut(a, n.B, n.P, 1, least);
  return a;
}
// Threads of the channels-last kernels that take part: a multiple of what makes a step whole points.
int active_threads(int C, int V) {
  int g = C, h = V;
  while (h != 0) { const int r = g % h; g = h; h = r; }
  const int unit = C / g;
  return unit <= kThreads ? kThreads / unit * unit : unit;
}

// scratch: sums of pieces, statistics or means
size_t norm_part_bytes(const NormShape& n) {
  const NormArgs f = n.last ? cut_points(n) : cut_groups(n), b = n.last ? f : cut_rows(n);
  const size_t fwd = (size_t)n.B * n.G * f.pieces, bwd = (size_t)n.B * n.C * b.pieces;
  return ((fwd > bwd ? fwd : bwd) * sizeof(double2) + 255) & ~size_t(255);
}

unsigned row_blocks(const NormArgs& a, bool short_rows) {
  const long long rows = (long long)a.B * a.C;
  return (unsigned)(short_rows ? (rows + kThreads / 64 - 1) / (kThreads / 64) : rows * a.pieces);
}

template <class T, int ACT>
hipError_t fwd(const NormShape& n, const T* x, const float* gamma, const float* beta, T* y, float* mean, float* rstd,
               void* ws, hipStream_t s) {
  double2* part = static_cast<double2*>(ws);
  Stat* stat = reinterpret_cast<Stat*>(static_cast<char*>(ws) + norm_part_bytes(n));
  const int bg = n.B * n.G;
  if (n.last) {
    const NormArgs a = cut_points(n);
    const int active = active_threads(n.C, kVec<T>), threads = (active + 63) / 64 * 64;
    hipLaunchKernelGGL((norm_last_sum_kernel<T>), dim3((unsigned)(n.B * a.pieces)), dim3(threads),
                       (size_t)active * kVec<T> * sizeof(double), s, a, active, x, reinterpret_cast<double*>(part));
    hipLaunchKernelGGL((norm_stat_kernel<T, true>), dim3(bg), dim3(kThreads), 0, s, a, x, part, stat, mean, rstd);
    if (n.P > 0)
      hipLaunchKernelGGL((norm_last_apply_kernel<T, ACT>), dim3((unsigned)(n.B * a.pieces)), dim3(threads), 0, s, a, active, x, gamma,
                         beta, stat, y);
    return hipGetLastError();
  }
  const NormArgs a = cut_groups(n), r = cut_rows(n);
  hipLaunchKernelGGL((norm_sum_kernel<T>), dim3((unsigned)(bg * a.pieces)), dim3(kThreads), 0, s, a, x, part);
  hipLaunchKernelGGL((norm_stat_kernel<T, false>), dim3(bg), dim3(kThreads), 0, s, a, x, part, stat, mean, rstd);
  if (n.P < kShortRow)
    hipLaunchKernelGGL((norm_apply_kernel<T, ACT, true>), dim3(row_blocks(r, true)), dim3(kThreads), 0, s, r, x, gamma, beta, stat, y);
  else
    hipLaunchKernelGGL((norm_apply_kernel<T, ACT, false>), dim3(row_blocks(r, false)), dim3(kThreads), 0, s, r, x, gamma, beta, stat, y);
  return hipGetLastError();
}

template <class T, int ACT>
hipError_t bwd(const NormShape& n, const T* x, const float* gamma, const float* beta, const float* mean, const float* rstd,
               const T* gy, T* gx, float* ggamma, float* gbeta, int accumulate, void* ws, hipStream_t s) {
  double2* part = static_cast<double2*>(ws);
  float2* m = reinterpret_cast<float2*>(static_cast<char*>(ws) + norm_part_bytes(n));
  const unsigned fold = (unsigned)(n.B * n.G + (n.C + kThreads / 64 - 1) / (kThreads / 64));
  if (n.last) {
    const NormArgs a = cut_points(n);
    const int active = active_threads(n.C, kVec<T>), threads = (active + 63) / 64 * 64;
    const dim3 grid((unsigned)(n.B * a.pieces));
    hipLaunchKernelGGL((norm_last_grad_sum_kernel<T, ACT>), grid, dim3(threads), (size_t)active * kVec<T> * sizeof(double), s, a, active,
                       x, gy, gamma, beta, mean, rstd, reinterpret_cast<double*>(part));
    hipLaunchKernelGGL(norm_grad_fold_kernel, dim3(fold), dim3(kThreads), 0, s, a, part, gamma, m, ggamma, gbeta, accumulate);
    if (gx != nullptr && n.P > 0)
      hipLaunchKernelGGL((norm_last_grad_apply_kernel<T, ACT>), grid, dim3(threads), 0, s, a, active, x, gy, gamma, beta, mean, rstd, m,
                         gx);
    return hipGetLastError();
  }
  const NormArgs r = cut_rows(n);
  const bool short_rows = n.P < kShortRow;
  const dim3 grid(row_blocks(r, short_rows));
  if (short_rows)
    hipLaunchKernelGGL((norm_grad_sum_kernel<T, ACT, true>), grid, dim3(kThreads), 0, s, r, x, gy, gamma, beta, mean, rstd, part);
  else
    hipLaunchKernelGGL((norm_grad_sum_kernel<T, ACT, false>), grid, dim3(kThreads), 0, s, r, x, gy, gamma, beta, mean, rstd, part);
  hipLaunchKernelGGL(norm_grad_fold_kernel, dim3(fold), dim3(kThreads), 0, s, r, part, gamma, m, ggamma, gbeta, accumulate);
  if (gx == nullptr) return hipGetLastError();
  if (short_rows)
    hipLaunchKernelGGL((norm_grad_apply_kernel<T, ACT, true>), grid, dim3(kThreads), 0, s, r, x, gy, gamma, beta, mean, rstd, m, gx);
  else
    hipLaunchKernelGGL((norm_grad_apply_kernel<T, ACT, false>), grid, dim3(kThreads), 0, s, r, x, gy, gamma, beta, mean, rstd, m, gx);
  return hipGetLastError();
}

// f(type, activation) for the type and activation of a descriptor
template <class F>
hipError_t dispatch(const NormShape& n, F&& f) {
  auto act = [&](auto t) {
    if (n.act == 1) return f(t, std::integral_constant<int, 1>());
    if (n.act == 2) return f(t, std::integral_constant<int, 2>());
    return f(t, std::integral_constant<int, 0>());
  };
  return n.bf16 ? act(u16()) : act(float());
}

}  // namespace

size_t group_norm_workspace_bytes(const NormShape& n) {
  return norm_part_bytes(n) + (((size_t)n.B * n.G * sizeof(Stat) + 255) & ~size_t(255));
}

hipError_t launch_group_norm_fwd(const NormShape& n, const void* x, const float* gamma, const float* beta, void* y,
                                 float* mean, float* rstd, void* ws, hipStream_t s) {
  return dispatch(n, [&](auto t, auto act) {
    typedef decltype(t) T;
    return fwd<T, decltype(act)::value>(n, static_cast<const T*>(x), gamma, beta, static_cast<T*>(y), mean, rstd, ws, s);
  });
}

hipError_t launch_group_norm_bwd(const NormShape& n, const void* x, const float* gamma, const float* beta, const float* mean,
                                 const float* rstd, const void* gy, void* gx, float* ggamma, float* gbeta, int accumulate,
                                 void* ws, hipStream_t s) {
  return dispatch(n, [&](auto t, auto act) {
    typedef decltype(t) T;
    return bwd<T, decltype(act)::value>(n, static_cast<const T*>(x), gamma, beta, mean, rstd, static_cast<const T*>(gy),
                                        static_cast<T*>(gx), ggamma, gbeta, accumulate, ws, s);
  });
}

}  // namespace fno
