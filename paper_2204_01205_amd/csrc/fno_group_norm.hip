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

// part[(bg, piece)] = (sum d, sum d^2); stat[bg].hi = k, for the launches that follow, which may write over x
template <class T>
__global__ __launch_bounds__(kThreads) void norm_sum_kernel(NormArgs a, const T* x, double2* part, Stat* stat) {
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
  if (threadIdx.x != 0) return;
  part[blockIdx.x] = make_double2(s, q);
  if (j == 0) stat[bg].hi = first;
}

// The statistics of group bg from its pieces' sums, in every thread of a block; red: as for block_sum2.
__device__ __forceinline__ Stat block_stat(const NormArgs& a, int pieces, const Stat* stat, const double2* part, long long bg,
                                           float* mean, float* rstd, double* red) {
  double s = 0.0, q = 0.0;
  for (int j = threadIdx.x; j < pieces; j += kThreads) {
    const double2 p = part[bg * pieces + j];
    s += p.x;
    q += p.y;
  }
  block_sum2(s, q, red);
  return stat_of(stat[bg].hi, s, q, a, mean, rstd, bg);
}

// Adds the pieces of every (b, g), a group a block.
__global__ __launch_bounds__(kThreads) void norm_stat_kernel(NormArgs a, const double2* part, Stat* stat, float* mean, float* rstd) {
  __shared__ double red[2 * kThreads / 64];
  const bool tells = threadIdx.x == 0;
  const Stat s = block_stat(a, a.pieces, stat, part, blockIdx.x, tells ? mean : nullptr, tells ? rstd : nullptr, red);
  __syncthreads();
  if (tells) stat[blockIdx.x] = s;
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

// A piece of a row per block; short: a row per wave.  part: the sums of the group's `parts` pieces, few enough for every
// block to add them itself (null: the statistics are in `stat`).
template <class T, int ACT, bool SHORT>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs a, const T* x, const float* gamma, const float* beta,
                                                              const Stat* stat, const double2* part, int parts, float* mean,
                                                              float* rstd, T* y) {
  __shared__ double red[2 * kThreads / 64];
  const long long row = SHORT ? (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6) : blockIdx.x / a.pieces;
  if (SHORT && row >= (long long)a.B * a.C) return;
  const int c = (int)(row % a.C);
  const long long j = SHORT ? 0 : blockIdx.x % a.pieces;
  Stat st;
  if (!SHORT && part != nullptr) {
    const bool tells = j == 0 && c % a.D == 0 && threadIdx.x == 0;
    st = block_stat(a, parts, stat, part, row / a.D, tells ? mean : nullptr, tells ? rstd : nullptr, red);
  } else {
    st = stat[row / a.D];
  }
  const Affine f = affine_of(st, gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
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

// A channel's parameter gradients, by a wave: sums over batch entries and pieces.  part[(b, c)][piece].
__device__ __forceinline__ void param_grads(const NormArgs& a, const double2* part, long long c, float* ggamma, float* gbeta,
                                            int accumulate) {
  if (c >= a.C) return;
  double s1 = 0.0, s2 = 0.0;
  const long long count = (long long)a.B * a.pieces;
  for (long long j = threadIdx.x & 63; j < count; j += 64) {
    const double2 p = part[(j / a.pieces * a.C + c) * a.pieces + j % a.pieces];
    s1 += p.x;
    s2 += p.y;
  }
  wave_sum2(s1, s2);
  if ((threadIdx.x & 63) != 0) return;
  if (gbeta != nullptr) gbeta[c] = (float)(accumulate ? (double)gbeta[c] + s1 : s1);
  if (ggamma != nullptr) ggamma[c] = (float)(accumulate ? (double)ggamma[c] + s2 : s2);
}
// A thread's share of the sums of gamma gz and gamma gz xh over a group: thread `tid` of `threads`
__device__ __forceinline__ void group_share(const NormArgs& a, const double2* part, const float* gamma, long long bg, int tid,
                                            int threads, double& s1, double& s2) {
  const long long count = (long long)a.D * a.pieces, at = bg * count;
  const int c0 = (int)(bg % a.G) * a.D;
  for (long long j = tid; j < count; j += threads) {
    const double2 p = part[at + j];
    const double ga = gamma ? gamma[c0 + (int)(j / a.pieces)] : 1.f;
    s1 = fma(ga, p.x, s1);
    s2 = fma(ga, p.y, s2);
  }
}

// Blocks 0 .. groups - 1 (B G, or none): m[bg] = the group's means of gamma gz and gamma gz xh.  The blocks behind: the
// parameters' gradients.
__global__ __launch_bounds__(kThreads) void norm_grad_fold_kernel(NormArgs a, unsigned groups, const double2* part,
                                                                  const float* gamma, float2* m, float* ggamma, float* gbeta,
                                                                  int accumulate) {
  __shared__ double red[2 * kThreads / 64];
  if (blockIdx.x >= groups)
    return param_grads(a, part, (long long)(blockIdx.x - groups) * (kThreads / 64) + (threadIdx.x >> 6), ggamma, gbeta, accumulate);
  double s1 = 0.0, s2 = 0.0;
  group_share(a, part, gamma, blockIdx.x, threadIdx.x, kThreads, s1, s2);
  block_sum2(s1, s2, red);
  if (threadIdx.x == 0) m[blockIdx.x] = make_float2((float)(s1 * a.inv_n), (float)(s2 * a.inv_n));
}

template <int ACT>
__device__ __forceinline__ float grad_of(const Slope& k, float2 m, float x, float gy) {
  float xh, gz;
  terms<ACT>(k, x, gy, xh, gz);
  return k.rstd * (fmaf(gz, k.gamma, -m.x) - xh * m.y);
}

// m null: every block adds its group's sums itself, and the blocks from `mine` on the parameters' gradients.
template <class T, int ACT, bool SHORT>
__global__ __launch_bounds__(kThreads) void norm_grad_apply_kernel(NormArgs a, unsigned mine, const T* x, const T* gy,
                                                                   const float* gamma, const float* beta, const float* mean,
                                                                   const float* rstd, const float2* m, const double2* part,
                                                                   float* ggamma, float* gbeta, int accumulate, T* gx) {
  constexpr int V = kVec<T>, U = 2;
  __shared__ double red[2 * kThreads / 64];
  if (!SHORT && blockIdx.x >= mine)
    return param_grads(a, part, (long long)(blockIdx.x - mine) * (kThreads / 64) + (threadIdx.x >> 6), ggamma, gbeta, accumulate);
  const long long row = SHORT ? (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6) : blockIdx.x / a.pieces;
  if (SHORT && row >= (long long)a.B * a.C) return;
  const int c = (int)(row % a.C);
  const long long bg = row / a.D;
  const Slope k{mean[bg], rstd[bg], gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f};
  float2 mm;
  if (SHORT || m != nullptr) {
    mm = m[bg];
  } else {
    double s1 = 0.0, s2 = 0.0;
    group_share(a, part, gamma, bg, threadIdx.x, kThreads, s1, s2);
    block_sum2(s1, s2, red);
    mm = make_float2((float)(s1 * a.inv_n), (float)(s2 * a.inv_n));
  }
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

// part[(b, g)][piece] = (sum d, sum d^2); stat[(b, g)].hi = k
template <class T>
__global__ __launch_bounds__(1024) void norm_last_sum_kernel(NormArgs a, int active, const T* x, double* part, Stat* stat) {
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
  if (j == 0)
    for (int g = threadIdx.x; g < a.G; g += blockDim.x) stat[(long long)b * a.G + g].hi = a.P > 0 ? load1(x + base + g * a.D) : 0.f;
}

// part: the sums of the batch entry's pieces, few enough for every block to add them itself, a group a wave (null: the
// statistics are in `stat`).
template <class T, int ACT>
__global__ __launch_bounds__(1024) void norm_last_apply_kernel(NormArgs a, int active, const T* x, const float* gamma,
                                                               const float* beta, const Stat* stat, const double2* part,
                                                               float* mean, float* rstd, T* y) {
  constexpr int V = kVec<T>, U = 4;
  extern __shared__ double lds[];
  const int b = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  Stat* const mine = reinterpret_cast<Stat*>(lds);
  if (part != nullptr) {
    const bool tells = j == 0 && (threadIdx.x & 63) == 0;
    for (int g = threadIdx.x >> 6; g < a.G; g += blockDim.x >> 6) {
      const long long bg = (long long)b * a.G + g;
      double s = 0.0, q = 0.0;
      for (int k = threadIdx.x & 63; k < a.pieces; k += 64) {
        const double2 p = part[bg * a.pieces + k];
        s += p.x;
        q += p.y;
      }
      wave_sum2(s, q);
      const Stat st = stat_of(stat[bg].hi, s, q, a, tells ? mean : nullptr, tells ? rstd : nullptr, bg);
      if ((threadIdx.x & 63) == 0) mine[g] = st;
    }
    __syncthreads();
  }
  const long long p0 = (long long)j * a.per, p1 = p0 + a.per < a.P ? p0 + a.per : a.P;
  const long long base = (long long)b * a.P * a.C;
  Affine f[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int c = ((int)threadIdx.x * V + u) % a.C;
    Stat st;
    if (part != nullptr) st = mine[c / a.D];
    else st = stat[(long long)b * a.G + c / a.D];
    f[u] = affine_of(st, gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
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
__global__ __launch_bounds__(1024) void norm_last_grad_apply_kernel(NormArgs a, unsigned mine, int active, const T* x, const T* gy,
                                                                    const float* gamma, const float* beta, const float* mean,
                                                                    const float* rstd, const float2* m, const double2* part,
                                                                    float* ggamma, float* gbeta, int accumulate, T* gx) {
  constexpr int V = kVec<T>, U = 2;
  extern __shared__ double lds[];
  if (blockIdx.x >= mine)
    return param_grads(a, part, (long long)(blockIdx.x - mine) * (blockDim.x >> 6) + (threadIdx.x >> 6), ggamma, gbeta, accumulate);
  float2* const own = reinterpret_cast<float2*>(lds);
  if (m == nullptr) {
    const long long b0 = blockIdx.x / a.pieces * (long long)a.G;
    for (int g = threadIdx.x >> 6; g < a.G; g += blockDim.x >> 6) {
      double s1 = 0.0, s2 = 0.0;
      group_share(a, part, gamma, b0 + g, threadIdx.x & 63, 64, s1, s2);
      wave_sum2(s1, s2);
      if ((threadIdx.x & 63) == 0) own[g] = make_float2((float)(s1 * a.inv_n), (float)(s2 * a.inv_n));
    }
    __syncthreads();
  }
  const int b = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  const long long p0 = (long long)j * a.per, p1 = p0 + a.per < a.P ? p0 + a.per : a.P;
  const long long base = (long long)b * a.P * a.C;
  Slope k[V];
  slopes_of<V>(a, b, gamma, beta, mean, rstd, k);
  float2 mm[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int g = (((int)threadIdx.x * V + u) % a.C) / a.D;
    if (m == nullptr) mm[u] = own[g];
    else mm[u] = m[(long long)b * a.G + g];
  }
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
// Groups that one block holds in its registers: one launch, x (and gy) read once.  A thread has 16 values of the group,
// those of whole 16-byte runs where the runs stay within a point's channels of the group (channels first: always), else
// every `threads`-th.  The adjoint's sums over a channel go through LDS.
// ------------------------------------------------------------------------------------------
constexpr int kSmallValues = 16;                          // of a thread
constexpr int kSmallFwd = 1024 * kSmallValues, kSmallBwd = 8192;

struct SmallArgs {
  int n;                // values of the group
  int run;              // 16-byte runs (1) or single values (0)
  unsigned by;          // 2^32 / (channels first: P, channels last: D) + 1, for divisions of numbers below 2^14; 0: by one
};
__device__ __forceinline__ int over(unsigned e, unsigned by) { return by == 0 ? (int)e : (int)__umulhi(e, by); }

// Calls f(k, e) for the thread's values, e their number in the group (below n).
template <class T, class F>
__device__ __forceinline__ void small_values(const SmallArgs& s, F&& f) {
  constexpr int V = kVec<T>;
#pragma unroll
  for (int k = 0; k < kSmallValues; ++k) {
    const int e = s.run ? ((k / V) * (int)blockDim.x + (int)threadIdx.x) * V + k % V : k * (int)blockDim.x + (int)threadIdx.x;
    if (e < s.n) f(k, e);
  }
}
template <bool LAST>
__device__ __forceinline__ long long small_at(const NormArgs& a, const SmallArgs& s, int b, int g, int e) {
  if (!LAST) return ((long long)b * a.C + (long long)g * a.D) * a.P + e;
  const int p = over(e, s.by);
  return ((long long)b * a.P + p) * a.C + g * a.D + (e - p * a.D);
}
template <bool LAST>
__device__ __forceinline__ int small_channel(const NormArgs& a, const SmallArgs& s, int e) {
  return LAST ? e - over(e, s.by) * a.D : over(e, s.by);
}
template <class T, bool LAST>
__device__ __forceinline__ void small_load(const NormArgs& a, const SmallArgs& s, int b, int g, const T* x, float (&v)[kSmallValues]) {
  constexpr int V = kVec<T>;
  if (s.run) {
    pack<T> q[kSmallValues / V];
#pragma unroll
    for (int k = 0; k < kSmallValues / V; ++k) {
      const int e = (k * (int)blockDim.x + (int)threadIdx.x) * V;
      q[k] = pack<T>{};
      if (e + V <= s.n) q[k] = load_any(x + small_at<LAST>(a, s, b, g, e));
    }
#pragma unroll
    for (int k = 0; k < kSmallValues / V; ++k) {
      float w[V];
      unpack(q[k], w);
#pragma unroll
      for (int u = 0; u < V; ++u) v[k * V + u] = w[u];
      const int e = (k * (int)blockDim.x + (int)threadIdx.x) * V;
      if (e < s.n && e + V > s.n) {                       // the group's last values, channels first
#pragma unroll
        for (int u = 0; u < V; ++u)
          if (e + u < s.n) v[k * V + u] = load1(x + small_at<LAST>(a, s, b, g, e + u));
      }
    }
    return;
  }
#pragma unroll
  for (int k = 0; k < kSmallValues; ++k) {
    const int e = k * (int)blockDim.x + (int)threadIdx.x;
    v[k] = e < s.n ? load1(x + small_at<LAST>(a, s, b, g, e)) : 0.f;
  }
}
template <class T, bool LAST>
__device__ __forceinline__ void small_store(const NormArgs& a, const SmallArgs& s, int b, int g, T* y, const float (&v)[kSmallValues]) {
  constexpr int V = kVec<T>;
  if (s.run) {
#pragma unroll
    for (int k = 0; k < kSmallValues / V; ++k) {
      const int e = (k * (int)blockDim.x + (int)threadIdx.x) * V;
      float w[V];
#pragma unroll
      for (int u = 0; u < V; ++u) w[u] = v[k * V + u];
      if (e + V <= s.n) {
        store_any(y + small_at<LAST>(a, s, b, g, e), repack(w));
      } else {
#pragma unroll
        for (int u = 0; u < V; ++u)
          if (e + u < s.n) store1(y + small_at<LAST>(a, s, b, g, e + u), w[u]);
      }
    }
    return;
  }
  small_values<T>(s, [&](int k, int e) { store1(y + small_at<LAST>(a, s, b, g, e), v[k]); });
}

template <class T, int ACT, bool LAST>
__global__ __launch_bounds__(1024) void norm_small_kernel(NormArgs a, SmallArgs s, const T* x, const float* gamma, const float* beta,
                                                          T* y, float* mean, float* rstd) {
  __shared__ double red[2 * 1024 / 64];
  __shared__ float2 affine[kMaxNormChannels];
  const int b = blockIdx.x / a.G, g = blockIdx.x % a.G;
  float v[kSmallValues];
  small_load<T, LAST>(a, s, b, g, x, v);
  const float first = load1(x + small_at<LAST>(a, s, b, g, 0));
  double sum = 0.0, square = 0.0;
  small_values<T>(s, [&](int k, int) {
    const double d = v[k] - first;
    sum += d;
    square = fma(d, d, square);
  });
  block_sum2(sum, square, red);
  const bool tells = threadIdx.x == 0;
  const Stat st = stat_of(first, sum, square, a, tells ? mean : nullptr, tells ? rstd : nullptr, blockIdx.x);
  for (int d = threadIdx.x; d < a.D; d += blockDim.x) {
    const Affine f = affine_of(st, gamma ? gamma[g * a.D + d] : 1.f, beta ? beta[g * a.D + d] : 0.f);
    affine[d] = make_float2(f.scale, f.shift);
  }
  __syncthreads();
  small_values<T>(s, [&](int k, int e) {
    const float2 f = affine[small_channel<LAST>(a, s, e)];
    v[k] = normed<ACT>(Affine{st.hi, f.x, f.y}, v[k]);
  });
  small_store<T, LAST>(a, s, b, g, y, v);
}

// part (B > 1) or ggamma and gbeta (B = 1) receive the channels' sums; lanes: how many add a channel's, a power of two.
template <class T, int ACT, bool LAST>
__global__ __launch_bounds__(1024) void norm_small_grad_kernel(NormArgs a, SmallArgs s, int lanes, const T* x, const T* gy,
                                                               const float* gamma, const float* beta, const float* mean,
                                                               const float* rstd, T* gx, double2* part, float* ggamma,
                                                               float* gbeta, int accumulate) {
  __shared__ double red[2 * 1024 / 64];
  __shared__ float2 affine[kMaxNormChannels];
  extern __shared__ double lds[];
  const int b = blockIdx.x / a.G, g = blockIdx.x % a.G;
  const bool params = part != nullptr || ggamma != nullptr || gbeta != nullptr;
  float v[kSmallValues], w[kSmallValues];
  small_load<T, LAST>(a, s, b, g, x, v);
  small_load<T, LAST>(a, s, b, g, gy, w);
  for (int d = threadIdx.x; d < a.D; d += blockDim.x)
    affine[d] = make_float2(gamma ? gamma[g * a.D + d] : 1.f, beta ? beta[g * a.D + d] : 0.f);
  const float mu = mean[blockIdx.x], rs = rstd[blockIdx.x];
  float2* const product = reinterpret_cast<float2*>(lds);      // gz and gz xh of every value
  __syncthreads();
  double s1 = 0.0, s2 = 0.0;
  small_values<T>(s, [&](int k, int e) {                  // v: xh, w: gamma gz
    const float2 f = affine[small_channel<LAST>(a, s, e)];
    float xh, gz;
    terms<ACT>(Slope{mu, rs, f.x, f.y}, v[k], w[k], xh, gz);
    v[k] = xh;
    w[k] = gz * f.x;
    s1 += w[k];
    s2 = fma((double)w[k], (double)xh, s2);
    if (params) product[e] = make_float2(gz, gz * xh);
  });
  block_sum2(s1, s2, red);
  if (gx != nullptr) {
    const float m1 = (float)(s1 * a.inv_n), m2 = (float)(s2 * a.inv_n);
    small_values<T>(s, [&](int k, int) { w[k] = rs * ((w[k] - m1) - v[k] * m2); });
    small_store<T, LAST>(a, s, b, g, gx, w);
  }
  if (!params) return;
  const int lane = threadIdx.x & (lanes - 1), P = (int)a.P;
  for (int d0 = 0; d0 < a.D; d0 += blockDim.x / lanes) {  // (the same number of turns for all lanes of a wave)
    const int d = d0 + threadIdx.x / lanes;
    double t1 = 0.0, t2 = 0.0;
    if (d < a.D)
      for (int p = lane; p < P; p += lanes) {
        const float2 q = product[LAST ? p * a.D + d : d * P + p];
        t1 += q.x;
        t2 += q.y;
      }
    for (int off = lanes >> 1; off >= 1; off >>= 1) {
      t1 += __shfl_xor(t1, off);
      t2 += __shfl_xor(t2, off);
    }
    if (d >= a.D || lane != 0) continue;
    const int c = g * a.D + d;
    if (part != nullptr) {
      part[(long long)b * a.C + c] = make_double2(t1, t2);
    } else {
      if (gbeta != nullptr) gbeta[c] = (float)(accumulate ? (double)gbeta[c] + t1 : t1);
      if (ggamma != nullptr) ggamma[c] = (float)(accumulate ? (double)ggamma[c] + t2 : t2);
    }
  }
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

// Sums of pieces that every block of the next launch adds itself (16 or 32 KB from the L2 a block), sparing a launch
constexpr long long kInlineParts = 1024;

bool small_fits(const NormShape& n, int most) { return n.P > 0 && n.P <= most && n.P * (n.C / n.G) <= most; }
SmallArgs small_args(const NormShape& n, int V) {
  const int D = n.C / n.G;
  const unsigned by = n.last ? (unsigned)D : (unsigned)n.P;
  return SmallArgs{(int)(n.P * D), !n.last || D % V == 0 ? 1 : 0, by == 1 ? 0u : (unsigned)(0x100000000ull / by) + 1u};
}
// Threads for n values, 4 of them at least a thread where there are enough waves, 16 at most.
int small_threads(int n) {
  const int t = (n + 3) / 4 < 256 ? (n + 3) / 4 : (n + kSmallValues - 1) / kSmallValues < 256 ? 256 : (n + kSmallValues - 1) / kSmallValues;
  return (t + 63) / 64 * 64;
}

template <class T, int ACT>
hipError_t fwd(const NormShape& n, const T* x, const float* gamma, const float* beta, T* y, float* mean, float* rstd,
               void* ws, hipStream_t s) {
  double2* part = static_cast<double2*>(ws);
  Stat* stat = reinterpret_cast<Stat*>(static_cast<char*>(ws) + norm_part_bytes(n));
  const int bg = n.B * n.G;
  if (small_fits(n, kSmallFwd)) {
    const NormArgs a = norm_args(n);
    const SmallArgs k = small_args(n, kVec<T>);
    if (n.last) hipLaunchKernelGGL((norm_small_kernel<T, ACT, true>), dim3(bg), dim3(small_threads(k.n)), 0, s, a, k, x, gamma, beta, y, mean, rstd);
    else hipLaunchKernelGGL((norm_small_kernel<T, ACT, false>), dim3(bg), dim3(small_threads(k.n)), 0, s, a, k, x, gamma, beta, y, mean, rstd);
    return hipGetLastError();
  }
  if (n.last) {
    const NormArgs a = cut_points(n);
    const int active = active_threads(n.C, kVec<T>), threads = (active + 63) / 64 * 64;
    const bool inside = (long long)n.G * a.pieces <= kInlineParts && n.P > 0;
    hipLaunchKernelGGL((norm_last_sum_kernel<T>), dim3((unsigned)(n.B * a.pieces)), dim3(threads),
                       (size_t)active * kVec<T> * sizeof(double), s, a, active, x, reinterpret_cast<double*>(part), stat);
    if (!inside) hipLaunchKernelGGL(norm_stat_kernel, dim3(bg), dim3(kThreads), 0, s, a, part, stat, mean, rstd);
    if (n.P > 0)
      hipLaunchKernelGGL((norm_last_apply_kernel<T, ACT>), dim3((unsigned)(n.B * a.pieces)), dim3(threads),
                         inside ? n.G * sizeof(Stat) : 0, s, a, active, x, gamma, beta, stat, inside ? part : nullptr, mean, rstd, y);
    return hipGetLastError();
  }
  const NormArgs a = cut_groups(n), r = cut_rows(n);
  const bool short_rows = n.P < kShortRow, inside = !short_rows && a.pieces <= kInlineParts / 4;
  hipLaunchKernelGGL((norm_sum_kernel<T>), dim3((unsigned)(bg * a.pieces)), dim3(kThreads), 0, s, a, x, part, stat);
  if (!inside) hipLaunchKernelGGL(norm_stat_kernel, dim3(bg), dim3(kThreads), 0, s, a, part, stat, mean, rstd);
  if (short_rows)
    hipLaunchKernelGGL((norm_apply_kernel<T, ACT, true>), dim3(row_blocks(r, true)), dim3(kThreads), 0, s, r, x, gamma, beta, stat,
                       nullptr, 0, mean, rstd, y);
  else
    hipLaunchKernelGGL((norm_apply_kernel<T, ACT, false>), dim3(row_blocks(r, false)), dim3(kThreads), 0, s, r, x, gamma, beta, stat,
                       inside ? part : nullptr, a.pieces, mean, rstd, y);
  return hipGetLastError();
}

template <class T, int ACT>
hipError_t bwd(const NormShape& n, const T* x, const float* gamma, const float* beta, const float* mean, const float* rstd,
               const T* gy, T* gx, float* ggamma, float* gbeta, int accumulate, void* ws, hipStream_t s) {
  double2* part = static_cast<double2*>(ws);
  float2* m = reinterpret_cast<float2*>(static_cast<char*>(ws) + norm_part_bytes(n));
  const bool params = ggamma != nullptr || gbeta != nullptr;
  if (small_fits(n, kSmallBwd)) {
    const NormArgs a = norm_args(n);
    const SmallArgs k = small_args(n, kVec<T>);
    int lanes = 1;
    while (lanes < 64 && lanes < n.P) lanes *= 2;
    const bool later = params && n.B > 1;
    const size_t lds = params ? k.n * sizeof(float2) : 0;
    auto launch = [&](auto last) {
      hipLaunchKernelGGL((norm_small_grad_kernel<T, ACT, decltype(last)::value>), dim3(n.B * n.G), dim3(small_threads(k.n)), lds, s, a, k,
                         lanes, x, gy, gamma, beta, mean, rstd, gx, later ? part : nullptr, ggamma, gbeta, accumulate);
    };
    if (n.last) launch(std::true_type());
    else launch(std::false_type());
    if (later)
      hipLaunchKernelGGL(norm_grad_fold_kernel, dim3((n.C + kThreads / 64 - 1) / (kThreads / 64)), dim3(kThreads), 0, s, a, 0u, part, gamma,
                         m, ggamma, gbeta, accumulate);
    return hipGetLastError();
  }
  const bool short_rows = !n.last && n.P < kShortRow;
  const NormArgs a = n.last ? cut_points(n) : cut_rows(n);
  const int active = active_threads(n.C, kVec<T>), threads = n.last ? (active + 63) / 64 * 64 : kThreads;
  const unsigned blocks = n.last ? (unsigned)(n.B * a.pieces) : row_blocks(a, short_rows);
  const unsigned channel_blocks = (unsigned)((n.C + threads / 64 - 1) / (threads / 64));
  if (n.last)
    hipLaunchKernelGGL((norm_last_grad_sum_kernel<T, ACT>), dim3(blocks), dim3(threads), (size_t)active * kVec<T> * sizeof(double), s, a,
                       active, x, gy, gamma, beta, mean, rstd, reinterpret_cast<double*>(part));
  else if (short_rows)
    hipLaunchKernelGGL((norm_grad_sum_kernel<T, ACT, true>), dim3(blocks), dim3(kThreads), 0, s, a, x, gy, gamma, beta, mean, rstd, part);
  else
    hipLaunchKernelGGL((norm_grad_sum_kernel<T, ACT, false>), dim3(blocks), dim3(kThreads), 0, s, a, x, gy, gamma, beta, mean, rstd, part);
  const bool writes = gx != nullptr && n.P > 0;
  const bool inside = writes && !short_rows && (long long)(n.last ? n.C : n.C / n.G) * a.pieces <= kInlineParts;
  if (!inside)
    hipLaunchKernelGGL(norm_grad_fold_kernel, dim3((unsigned)(n.B * n.G) + (n.C + kThreads / 64 - 1) / (kThreads / 64)), dim3(kThreads), 0, s,
                       a, (unsigned)(n.B * n.G), part, gamma, m, ggamma, gbeta, accumulate);
  if (!writes) return hipGetLastError();
  const dim3 grid(blocks + (inside && params ? channel_blocks : 0));
  const float2* means = inside ? nullptr : m;
  if (n.last)
    hipLaunchKernelGGL((norm_last_grad_apply_kernel<T, ACT>), grid, dim3(threads), inside ? n.G * sizeof(float2) : 0, s, a, blocks, active,
                       x, gy, gamma, beta, mean, rstd, means, part, ggamma, gbeta, accumulate, gx);
  else if (short_rows)
    hipLaunchKernelGGL((norm_grad_apply_kernel<T, ACT, true>), grid, dim3(kThreads), 0, s, a, blocks, x, gy, gamma, beta, mean, rstd, means,
                       part, ggamma, gbeta, accumulate, gx);
  else
    hipLaunchKernelGGL((norm_grad_apply_kernel<T, ACT, false>), grid, dim3(kThreads), 0, s, a, blocks, x, gy, gamma, beta, mean, rstd, means,
                       part, ggamma, gbeta, accumulate, gx);
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
