// Group norm with an activation, forward and adjoint, over fields [B][C][P] (channels first) or [B][P][C] (channels
// last) in float or bf16.
//
// What the operator moves bounds it: x in and y out (adjoint: x and gy in, gx out), 20 to 40 operations a value.  The
// statistics (adjoint: the sums) of a group need all of it before its first output, so a group that does not fit one
// block's registers is read twice: sums of pieces, a small launch that adds the pieces' sums in a fixed order, and the
// sweep that writes.
//
// Statistics: a block takes mean and variance of its piece from d = x - k, mean = k + E d, var = E d^2 - (E d)^2, k the piece's
// first value (of the group), and the pieces are put together by var = E (var_j + (mean_j - mean)^2), about the mean of the first
// one.  k is one of the N values it is subtracted from, so that (E d)^2 <= N var: what the subtraction of the squares can lose is a
// factor N of a piece, which double has to spare, whatever k is and wherever the group lies (with the squares in float, a
// constant field with zeros at its corners had rstd off by 1e-2).  Differences and squares are formed in double too: no float
// is too large or too small for them.  Adjoint: four or eight terms are added in float, everything else in double.
//
// Measured, with the bytes that the launches move (x twice; adjoint x and gy twice) at a copy's 6.2 TB/s in brackets: 60 x 60 x
// 64 x 30 points, 20 channels, forward 270 us (268); 64 x 64 x 64 x 20, 32 channels last, 330 (325); 128 x 128 x 64 x 32, 20
// channels, adjoint 2.12 ms (2.16).  bf16, adjoint of 2 x 64 x 64 x 64 x 16, 20 channels last: 340 us (270), the vector unit has
// 27 and 28 instructions a value, two of them transcendental, and is busy for 125 of 171 us and 128 of 208.  Fields of a few MB:
// launches of 4 to 13 us each.
#include "fno_norm_device.h"

#include <climits>
#include <type_traits>

namespace fno {

namespace {

struct NormArgs {
  int B, C, G, D;       // D = C / G
  long long P;
  double inv_n, eps;    // inv_n = 1 / (D P)
  // A range (forward, channels first: a group; adjoint, channels first: a row; channels last: a batch entry) is cut into
  // tiles of 16 KB.  The launches that write take a tile a block, or deal the tiles to the blocks in turn, so that all blocks
  // together move through memory in one window (128 x 128 x 64 x 32, 20 channels, adjoint: 1.31 ms, 1.70 with a stretch of
  // tiles for every block); those that only read take a stretch each (the same: 0.86 ms, 0.95 in turn).
  int pieces;           // blocks of a range
  int run;              // tiles of a stretch
};
// How ranges were cut into pieces for the statistics.  A range: channels first the values of a group, channels last all of a
// batch entry; begin: where it starts, counted from an aligned base.
struct Cut {
  long long range, stretch;      // values of a range, and of a piece
  double inv;                    // 1 / range
  int pieces;
  int align;                     // pieces start at multiples of this; what lies before and behind belongs to the first one
};
__device__ __forceinline__ long long piece_values(const Cut& c, long long begin, int j) {
  long long head = -begin & (c.align - 1);
  if (head > c.range) head = c.range;
  const long long whole = (c.range - head) & -(long long)c.align;
  long long v = whole - j * c.stretch;
  v = v < 0 ? 0 : v > c.stretch ? c.stretch : v;
  return j == 0 ? v + (c.range - whole) : v;
}

// What a group's values go through: xh = (x - mean) rstd with the mean in two floats, so that x - hi is exact near it.
struct Stat {
  float hi, lo, rstd, pad;
};
// mean and variance of values of which d = x - k has the mean `off` and d^2 the mean `square`
__device__ __forceinline__ double2 moments_of(double k, double off, double square) {
  const double var = square - off * off;
  return make_double2(k + off, var < 0.0 ? 0.0 : var);   // (a NaN stays one)
}
__device__ __forceinline__ Stat stat_of(double2 moments, double eps, float* mean, float* rstd, long long at) {
  const double mu = moments.x, rs = 1.0 / sqrt(moments.y + eps);
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

// The 16-byte pieces of [begin, end) that start at multiples of their length go in tiles of U pieces a thread, of which this
// call takes number `tile` and every `stride`-th after it, `count` at most: vecs(at, step) for a whole tile, vec(at) for the
// pieces of the last one, and, with tile 0, one(at) for the values before and behind the pieces.  Places count from a 16-byte
// aligned base.
template <int V, int U, class FVecs, class FVec, class FOne>
__device__ __forceinline__ void sweep(long long begin, long long end, int tid, int threads, long long tile, long long stride,
                                      int count, FVecs&& vecs, FVec&& vec, FOne&& one) {
  long long lo = (begin + V - 1) / V * V;
  if (lo > end) lo = end;
  const long long hi = lo + (end - lo) / V * V, step = (long long)threads * V, size = step * U;
  long long base = lo + tile * size;
  for (int i = 0; i < count && base < hi; ++i, base += stride * size) {
    const long long at = base + (long long)tid * V;
    if (base + size <= hi) {
      vecs(at, step);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (at + u * step < hi) vec(at + u * step);
    }
  }
  if (tile != 0) return;
  if (begin + tid < lo) one(begin + tid);
  if (hi + tid < end) one(hi + tid);
}

// ------------------------------------------------------------------------------------------
// Channels first.  A group's values lie together: pieces of them whatever the channel for the statistics; a block's
// piece of one row (one channel), or whole short rows wave by wave, where gamma and beta come in.
// ------------------------------------------------------------------------------------------

// part[(bg, piece)] = mean and variance of the piece's values
template <class T, bool STREAM>
__global__ __launch_bounds__(kThreads) void norm_sum_kernel(NormArgs a, Cut cut, const T* x, double2* part) {
  constexpr int V = kVec<T>, U = 4;
  __shared__ double red[2 * kThreads / 64];
  const long long bg = blockIdx.x / a.pieces, begin = bg * cut.range;
  const int j = blockIdx.x % a.pieces;
  const long long count = piece_values(cut, begin, j);
  const double k = count > 0 ? load1(x + (j == 0 ? begin : (begin + V - 1) / V * V + j * cut.stretch)) : 0.f;
  double s = 0.0, q = 0.0;
  auto add1 = [&](float v) {
    const double d = v - k;
    s += d;
    q = fma(d, d, q);
  };
  auto add = [&](pack<T> p) {
    float v[V];
    unpack(p, v);
#pragma unroll
    for (int u = 0; u < V; ++u) add1(v[u]);
  };
  sweep<V, U>(begin, begin + cut.range, threadIdx.x, kThreads, (long long)j * a.run, 1, a.run,
              [&](long long at, long long step) {
                pack<T> p[U];
#pragma unroll
                for (int u = 0; u < U; ++u) p[u] = load_pack<STREAM>(x + at + u * step);
#pragma unroll
                for (int u = 0; u < U; ++u) add(p[u]);
              },
              [&](long long at) { add(load_pack<STREAM>(x + at)); },
              [&](long long at) { add1(load1(x + at)); });
  block_sum2(s, q, red);
  const double inv = count > 0 ? 1.0 / (double)count : 0.0;
  if (threadIdx.x == 0) part[bg * a.pieces + j] = moments_of(k, s * inv, q * inv);
}

// A thread's share of the sums that give a range's moments about the mean of its first piece; part: the range's pieces.
__device__ __forceinline__ void piece_share(const Cut& c, long long begin, const double2* part, int tid, int threads, double& s,
                                            double& q) {
  const double k = part[0].x;
  for (int j = tid; j < c.pieces; j += threads) {
    const double2 p = part[j];
    const double w = (double)piece_values(c, begin, j), d = p.x - k;
    s = fma(w, d, s);
    q = fma(w, fma(d, d, p.y), q);
  }
}
// The statistics of group bg from its pieces, in every thread of a block; red: as for block_sum2.
__device__ __forceinline__ Stat block_stat(const NormArgs& a, const Cut& c, long long begin, const double2* part, long long bg,
                                           float* mean, float* rstd, double* red) {
  double s = 0.0, q = 0.0;
  part += bg * c.pieces;
  piece_share(c, begin, part, threadIdx.x, kThreads, s, q);
  block_sum2(s, q, red);
  return stat_of(moments_of(part[0].x, s * c.inv, q * c.inv), a.eps, mean, rstd, bg);
}

// Puts the pieces of every (b, g) together, a group a block.
__global__ __launch_bounds__(kThreads) void norm_stat_kernel(NormArgs a, Cut cut, const double2* part, Stat* stat, float* mean,
                                                             float* rstd) {
  __shared__ double red[2 * kThreads / 64];
  const bool tells = threadIdx.x == 0;
  const long long bg = blockIdx.x;
  const Stat s = block_stat(a, cut, bg * cut.range, part, bg, tells ? mean : nullptr, tells ? rstd : nullptr, red);
  if (tells) stat[bg] = s;
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

template <class T, int ACT, bool STREAM>
__device__ __forceinline__ void apply_range(const Affine& f, const T* x, T* y, long long begin, long long end, int tid, int threads,
                                            long long tile, long long stride) {
  constexpr int V = kVec<T>, U = 4;
  auto put = [&](long long at, pack<T> k) {
    float v[V];
    unpack(k, v);
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = normed<ACT>(f, v[u]);
    store_pack<STREAM>(y + at, repack(v));
  };
  sweep<V, U>(begin, end, tid, threads, tile, stride, INT_MAX,
              [&](long long at, long long step) {
                pack<T> k[U];
#pragma unroll
                for (int u = 0; u < U; ++u) k[u] = load_pack<STREAM>(x + at + u * step);
#pragma unroll
                for (int u = 0; u < U; ++u) put(at + u * step, k[u]);
              },
              [&](long long at) { put(at, load_pack<STREAM>(x + at)); },
              [&](long long at) { store1(y + at, normed<ACT>(f, load1(x + at))); });
}

// A piece of a row per block; short: a row per wave.  part: the moments of the groups' pieces, few enough for every block to put
// its group's together itself (null: the statistics are in `stat`).
template <class T, int ACT, bool SHORT, bool STREAM>
__global__ __launch_bounds__(kThreads) void norm_apply_kernel(NormArgs a, const T* x, const float* gamma, const float* beta,
                                                              const Stat* stat, const double2* part, Cut cut, float* mean,
                                                              float* rstd, T* y) {
  __shared__ double red[2 * kThreads / 64];
  const long long row = SHORT ? (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6) : blockIdx.x / a.pieces;
  if (SHORT && row >= (long long)a.B * a.C) return;
  const int c = (int)(row % a.C);
  const long long j = SHORT ? 0 : blockIdx.x % a.pieces;
  Stat st;
  if (!SHORT && part != nullptr) {
    const bool tells = j == 0 && c % a.D == 0 && threadIdx.x == 0;
    st = block_stat(a, cut, row / a.D * cut.range, part, row / a.D, tells ? mean : nullptr, tells ? rstd : nullptr, red);
  } else {
    st = stat[row / a.D];
  }
  const Affine f = affine_of(st, gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
  if (SHORT) apply_range<T, ACT, STREAM>(f, x, y, row * a.P, (row + 1) * a.P, threadIdx.x & 63, 64, 0, 1);
  else apply_range<T, ACT, STREAM>(f, x, y, row * a.P, (row + 1) * a.P, threadIdx.x, kThreads, j, a.pieces);
}

// What one channel's values go through in the adjoint: d = x - mean, gz = gy act'(d rstd gamma + beta)
struct Slope {
  float mean, scale, shift;    // rstd gamma and beta in units of the activation's slope
};
template <int ACT>
__device__ __forceinline__ Slope slope_of(float mean, float rstd, float gamma, float beta) {
  return Slope{mean, rstd * gamma * kArg<ACT>, beta * kArg<ACT>};
}
template <int ACT>
__device__ __forceinline__ void terms(const Slope& k, float x, float gy, float& d, float& gz) {
  d = x - k.mean;
  gz = ACT == 0 ? gy : gy * slope_f<ACT>(fmaf(d, k.scale, k.shift));
}
// and gx = gz rstd gamma - rstd m1 - xh rstd m2, m1 and m2 the group's means of gamma gz and gamma gz xh.  (xh = d rstd costs a
// product a value; rstd^2 m2 in its place, for d, would leave the floats where rstd is past 1e18 or below 1e-18.)
struct Weights {
  float rstd, gz, xh, one;
};
__device__ __forceinline__ Weights weights_of(float rstd, float gamma, float2 m) {
  return Weights{rstd, rstd * gamma, -rstd * m.y, -rstd * m.x};
}
template <int ACT>
__device__ __forceinline__ float grad_of(const Slope& k, const Weights& w, float x, float gy) {
  float d, gz;
  terms<ACT>(k, x, gy, d, gz);
  return fmaf(gz, w.gz, fmaf(d * w.rstd, w.xh, w.one));
}

// part[(row, piece)] = (sum gz, sum gz xh)
template <class T, int ACT, bool SHORT, bool STREAM>
__global__ __launch_bounds__(kThreads) void norm_grad_sum_kernel(NormArgs a, const T* x, const T* gy, const float* gamma,
                                                                 const float* beta, const float* mean, const float* rstd,
                                                                 double2* part) {
  constexpr int V = kVec<T>, U = 2;
  __shared__ double red[2 * kThreads / 64];
  const long long row = SHORT ? (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6) : blockIdx.x / a.pieces;
  if (SHORT && row >= (long long)a.B * a.C) return;
  const int c = (int)(row % a.C);
  const long long bg = row / a.D;
  const float rs = rstd[bg], ga = gamma ? gamma[c] : 1.f;
  const Slope k = slope_of<ACT>(mean[bg], rs, ga, beta ? beta[c] : 0.f);
  const long long j = SHORT ? 0 : blockIdx.x % a.pieces;
  double s1 = 0.0, s2 = 0.0;
  auto add = [&](pack<T> px, pack<T> pg) {
    float v[V], g[V], t1 = 0.f, t2 = 0.f;
    unpack(px, v);
    unpack(pg, g);
#pragma unroll
    for (int u = 0; u < V; ++u) {
      float d, gz;
      terms<ACT>(k, v[u], g[u], d, gz);
      t1 += gz;
      t2 = fmaf(gz, d, t2);
    }
    s1 += t1;                                            // 4 or 8 terms in float, then doubles
    s2 += t2;
  };
  sweep<V, U>(row * a.P, (row + 1) * a.P, SHORT ? threadIdx.x & 63 : threadIdx.x, SHORT ? 64 : kThreads,
              SHORT ? 0 : j * a.run, 1, SHORT ? INT_MAX : a.run,
              [&](long long at, long long step) {
                pack<T> px[U], pg[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                  px[u] = load_pack<STREAM>(x + at + u * step);
                  pg[u] = load_pack<STREAM>(gy + at + u * step);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) add(px[u], pg[u]);
              },
              [&](long long at) { add(load_pack<STREAM>(x + at), load_pack<STREAM>(gy + at)); },
              [&](long long at) {
                float d, gz;
                terms<ACT>(k, load1(x + at), load1(gy + at), d, gz);
                s1 += gz;
                s2 = fma((double)gz, (double)d, s2);
              });
  if (SHORT) {
    wave_sum2(s1, s2);
    if ((threadIdx.x & 63) == 0) part[row] = make_double2(s1, s2 * rs);
  } else {
    block_sum2(s1, s2, red);
    if (threadIdx.x == 0) part[row * a.pieces + j] = make_double2(s1, s2 * rs);
  }
}

// A thread's share of a channel's parameter gradients: sums over batch entries and pieces.  part[(b, c)][piece].
__device__ __forceinline__ void channel_share(const NormArgs& a, int pieces, const double2* part, long long c, int tid, int threads,
                                              double& s1, double& s2) {
  const int count = a.B * pieces;
#pragma unroll 8
  for (int q = tid; q < count; q += threads) {
    const int b = q / pieces;
    const double2 p = part[((long long)b * a.C + c) * pieces + (q - b * pieces)];
    s1 += p.x;
    s2 += p.y;
  }
}
__device__ __forceinline__ void put_params(long long c, double s1, double s2, float* ggamma, float* gbeta, int accumulate) {
  if (gbeta != nullptr) gbeta[c] = (float)(accumulate ? (double)gbeta[c] + s1 : s1);
  if (ggamma != nullptr) ggamma[c] = (float)(accumulate ? (double)ggamma[c] + s2 : s2);
}
// The whole of it, by a wave
__device__ __forceinline__ void param_grads(const NormArgs& a, int pieces, const double2* part, long long c, float* ggamma,
                                            float* gbeta, int accumulate) {
  if (c >= a.C) return;
  double s1 = 0.0, s2 = 0.0;
  channel_share(a, pieces, part, c, threadIdx.x & 63, 64, s1, s2);
  wave_sum2(s1, s2);
  if ((threadIdx.x & 63) == 0) put_params(c, s1, s2, ggamma, gbeta, accumulate);
}
// A thread's share of the sums of gamma gz and gamma gz xh over a group: thread `tid` of `threads`
__device__ __forceinline__ void group_share(const NormArgs& a, int pieces, const double2* part, const float* gamma, long long bg,
                                            int tid, int threads, double& s1, double& s2) {
  const double2* const at = part + bg * a.D * pieces;
  const int c0 = (int)(bg % a.G) * a.D;
  if (pieces >= threads) {
    for (int d = 0; d < a.D; ++d) {
      const double ga = gamma ? gamma[c0 + d] : 1.f;
#pragma unroll 8
      for (int j = tid; j < pieces; j += threads) {
        const double2 p = at[(long long)d * pieces + j];
        s1 = fma(ga, p.x, s1);
        s2 = fma(ga, p.y, s2);
      }
    }
  } else {
#pragma unroll 4
    for (int j = tid; j < a.D * pieces; j += threads) {
      const double2 p = at[j];
      const double ga = gamma ? gamma[c0 + j / pieces] : 1.f;
      s1 = fma(ga, p.x, s1);
      s2 = fma(ga, p.y, s2);
    }
  }
}

constexpr int kFoldThreads = 1024;     // one block has a group's tens of thousands of sums to add
// Groups, or channels, of a block that have this many sums each: one, or, where they are few, a wave each.  (Groups are many only
// where their sums are few: with 2^22 groups there are 2 a group, and a block for each would be more threads than a launch has.)
// Adjoint, us, now, a block each, a wave each: 64 x 64 groups of 9000 values 124, 147, 124; one group of 1024 rows of 20000 81.6,
// 85.7, 99.0; channels last, 64 x 128 groups of 3000 95.6, 139.7, 100.5.
__host__ __device__ __forceinline__ int fold_each(int sums) { return sums <= 512 ? kFoldThreads / 64 : 1; }
// Blocks 0 .. blocks - 1 (maybe none): m[bg] = the group's means of gamma gz and gamma gz xh.  The blocks behind: the parameter
// gradients.
__global__ __launch_bounds__(kFoldThreads) void norm_grad_fold_kernel(NormArgs a, unsigned blocks, const double2* part,
                                                                      const float* gamma, float2* m, float* ggamma, float* gbeta,
                                                                      int accumulate) {
  __shared__ double red[2 * kFoldThreads / 64];
  double s1 = 0.0, s2 = 0.0;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (blockIdx.x >= blocks) {
    const unsigned at = blockIdx.x - blocks;
    if (fold_each(a.B * a.pieces) > 1)
      return param_grads(a, a.pieces, part, (long long)at * (kFoldThreads / 64) + wave, ggamma, gbeta, accumulate);
    channel_share(a, a.pieces, part, at, threadIdx.x, kFoldThreads, s1, s2);
    block_sum2(s1, s2, red);
    if (threadIdx.x == 0) put_params(at, s1, s2, ggamma, gbeta, accumulate);
    return;
  }
  if (fold_each(a.D * a.pieces) > 1) {
    const long long bg = (long long)blockIdx.x * (kFoldThreads / 64) + wave;
    if (bg >= (long long)a.B * a.G) return;
    group_share(a, a.pieces, part, gamma, bg, lane, 64, s1, s2);
    wave_sum2(s1, s2);
    if (lane == 0) m[bg] = make_float2((float)(s1 * a.inv_n), (float)(s2 * a.inv_n));
    return;
  }
  group_share(a, a.pieces, part, gamma, blockIdx.x, threadIdx.x, kFoldThreads, s1, s2);
  block_sum2(s1, s2, red);
  if (threadIdx.x == 0) m[blockIdx.x] = make_float2((float)(s1 * a.inv_n), (float)(s2 * a.inv_n));
}

// m null: every block adds its group's sums itself, and the blocks from `mine` on the parameters' gradients.
template <class T, int ACT, bool SHORT, bool STREAM>
__global__ __launch_bounds__(kThreads) void norm_grad_apply_kernel(NormArgs a, unsigned mine, const T* x, const T* gy,
                                                                   const float* gamma, const float* beta, const float* mean,
                                                                   const float* rstd, const float2* m, const double2* part, int parts,
                                                                   float* ggamma, float* gbeta, int accumulate, T* gx) {
  constexpr int V = kVec<T>, U = 2;
  __shared__ double red[2 * kThreads / 64];
  if (!SHORT && blockIdx.x >= mine)
    return param_grads(a, parts, part, (long long)(blockIdx.x - mine) * (kThreads / 64) + (threadIdx.x >> 6), ggamma, gbeta,
                       accumulate);
  const long long row = SHORT ? (long long)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6) : blockIdx.x / a.pieces;
  if (SHORT && row >= (long long)a.B * a.C) return;
  const int c = (int)(row % a.C);
  const long long bg = row / a.D;
  const float rs = rstd[bg], ga = gamma ? gamma[c] : 1.f;
  const Slope k = slope_of<ACT>(mean[bg], rs, ga, beta ? beta[c] : 0.f);
  float2 mm;
  if (SHORT || m != nullptr) {
    mm = m[bg];
  } else {
    double s1 = 0.0, s2 = 0.0;
    group_share(a, parts, part, gamma, bg, threadIdx.x, kThreads, s1, s2);
    block_sum2(s1, s2, red);
    mm = make_float2((float)(s1 * a.inv_n), (float)(s2 * a.inv_n));
  }
  const long long j = SHORT ? 0 : blockIdx.x % a.pieces;
  const Weights w = weights_of(rs, ga, mm);
  auto put = [&](long long at, pack<T> px, pack<T> pg) {
    float v[V], g[V];
    unpack(px, v);
    unpack(pg, g);
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = grad_of<ACT>(k, w, v[u], g[u]);
    store_pack<STREAM>(gx + at, repack(v));
  };
  sweep<V, U>(row * a.P, (row + 1) * a.P, SHORT ? threadIdx.x & 63 : threadIdx.x, SHORT ? 64 : kThreads, j, a.pieces,
              INT_MAX,
              [&](long long at, long long step) {
                pack<T> px[U], pg[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                  px[u] = load_pack<STREAM>(x + at + u * step);
                  pg[u] = load_pack<STREAM>(gy + at + u * step);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) put(at + u * step, px[u], pg[u]);
              },
              [&](long long at) { put(at, load_pack<STREAM>(x + at), load_pack<STREAM>(gy + at)); },
              [&](long long at) { store1(gx + at, grad_of<ACT>(k, w, load1(x + at), load1(gy + at))); });
}

// ------------------------------------------------------------------------------------------
// Channels last.  The points of a batch entry lie one behind the other, C values each.  `active` threads take 16 bytes each,
// one behind the other; active x V is a multiple of C, so that a thread meets the same V channels in every step: their
// factors and sums stay in its registers, and no access knows of channels.  Batch entries whose start is not 16-byte
// aligned are read and written in 16-byte accesses at their values' own alignment.
// ------------------------------------------------------------------------------------------

template <bool STREAM, class T>
__device__ __forceinline__ pack<T> load_any(const T* p) {
  typedef pack<T> loose __attribute__((aligned(sizeof(T))));
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const loose*>(p));
  else return *reinterpret_cast<const loose*>(p);
}
template <bool STREAM, class T>
__device__ __forceinline__ void store_any(T* p, pack<T> v) {
  typedef pack<T> loose __attribute__((aligned(sizeof(T))));
  if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<loose*>(p));
  else *reinterpret_cast<loose*>(p) = v;
}

// The values [begin, end) of whole points, as sweep() does; one(at, u) for the last values, which do not fill 16 bytes (u:
// which of the thread's channels).
template <int V, int U, class FVecs, class FVec, class FOne>
__device__ __forceinline__ void sweep_last(long long begin, long long end, int active, long long tile, long long stride, int count,
                                           FVecs&& vecs, FVec&& vec, FOne&& one) {
  if ((int)threadIdx.x >= active) return;
  const long long step = (long long)active * V, size = step * U;
  long long base = begin + tile * size;
  for (int i = 0; i < count && base < end; ++i, base += stride * size) {
    long long at = base + (long long)threadIdx.x * V;
    if (base + size <= end) {
      vecs(at, step);
    } else {
      for (; at + V <= end; at += step) vec(at);
#pragma unroll
      for (int u = 0; u < V; ++u)
        if (at + u < end) one(at + u, u);
    }
  }
}

// Adds the pairs of a block's threads by channel: lds[r C + c], r < rows, as every active thread left its V behind those of the
// thread before.  First k threads for every channel, then their k sums in turn or, where they are many, as a tree.  Returns
// where the C sums are, in front of every thread.
__device__ __forceinline__ double2* channel_sums(double2* lds, int rows, int C) {
  double2* const sums = lds + rows * C;
  int k = (int)blockDim.x / C;
  if (k < 1) k = 1;
  if (k > rows) k = rows;
  __syncthreads();
  for (int t = threadIdx.x; t < C * k; t += blockDim.x) {
    const int c = t % C;
    double2 s = make_double2(0.0, 0.0);
    for (int r = t / C; r < rows; r += k) {
      s.x += lds[r * C + c].x;
      s.y += lds[r * C + c].y;
    }
    sums[t] = s;
  }
  __syncthreads();
  while (k > 16) {
    const int h = (k + 1) >> 1;
    for (int t = threadIdx.x; t < (k - h) * C; t += blockDim.x) {
      sums[t].x += sums[t + h * C].x;
      sums[t].y += sums[t + h * C].y;
    }
    k = h;
    __syncthreads();
  }
  if (k > 1) {
    for (int c = threadIdx.x; c < C; c += blockDim.x) {
      double2 s = sums[c];
      for (int r = 1; r < k; ++r) {
        s.x += sums[r * C + c].x;
        s.y += sums[r * C + c].y;
      }
      sums[c] = s;
    }
    __syncthreads();
  }
  return sums;
}

// part[(b, g)][piece] = mean and variance of the group's values in the piece
template <class T, bool STREAM>
__global__ __launch_bounds__(1024) void norm_last_sum_kernel(NormArgs a, Cut cut, int active, const T* x, double2* part) {
  constexpr int V = kVec<T>, U = 4;
  extern __shared__ double2 pairs[];
  __shared__ float firsts[kMaxNormChannels];
  const int b = (int)blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  const long long base = (long long)b * cut.range;
  const double count = (double)(piece_values(cut, 0, j) / a.G);        // of every group
  double s[V], q[V], k[V];
  for (int g = threadIdx.x; g < a.G; g += blockDim.x) firsts[g] = count > 0.0 ? load1(x + base + j * cut.stretch + g * a.D) : 0.f;
  __syncthreads();
#pragma unroll
  for (int u = 0; u < V; ++u) {
    s[u] = q[u] = 0.0;
    k[u] = firsts[((int)threadIdx.x * V + u) % a.C / a.D];
  }
  auto add1 = [&](int u, float v) {
    const double d = v - k[u];
    s[u] += d;
    q[u] = fma(d, d, q[u]);
  };
  auto add = [&](pack<T> p) {
    float v[V];
    unpack(p, v);
#pragma unroll
    for (int u = 0; u < V; ++u) add1(u, v[u]);
  };
  sweep_last<V, U>(base, base + cut.range, active, (long long)j * a.run, 1, a.run,
                   [&](long long at, long long step) {
                     pack<T> p[U];
#pragma unroll
                     for (int u = 0; u < U; ++u) p[u] = load_any<STREAM>(x + at + u * step);
#pragma unroll
                     for (int u = 0; u < U; ++u) add(p[u]);
                   },
                   [&](long long at) { add(load_any<STREAM>(x + at)); },
                   [&](long long at, int u) {
                     const float v = load1(x + at);
#pragma unroll
                     for (int w = 0; w < V; ++w)
                       if (w == u) add1(w, v);
                   });
  if ((int)threadIdx.x < active) {
#pragma unroll
    for (int u = 0; u < V; ++u) pairs[threadIdx.x * V + u] = make_double2(s[u], q[u]);
  }
  const double2* const sums = channel_sums(pairs, active * V / a.C, a.C);
  double2* const to = part + (long long)b * a.G * a.pieces + j;
  const double inv = count > 0.0 ? 1.0 / count : 0.0;
  auto put = [&](int g, double2 m) { to[(long long)g * a.pieces] = moments_of(firsts[g], m.x * inv, m.y * inv); };
  // a group a thread, or a wave (forward, us: 64 groups of one channel 12.2 and 18.7, 8 of 8 12.1 and 12.6, 4 of 32 12.2 and 12.0, one
  // of 1024 27.7 and 17.5)
  if (a.D <= 32) {
    for (int g = threadIdx.x; g < a.G; g += blockDim.x) {
      double2 m = sums[g * a.D];
      for (int d = 1; d < a.D; ++d) {
        m.x += sums[g * a.D + d].x;
        m.y += sums[g * a.D + d].y;
      }
      put(g, m);
    }
  } else {
    for (int g = threadIdx.x >> 6; g < a.G; g += blockDim.x >> 6) {
      double2 m = make_double2(0.0, 0.0);
      for (int d = threadIdx.x & 63; d < a.D; d += 64) {
        m.x += sums[g * a.D + d].x;
        m.y += sums[g * a.D + d].y;
      }
      wave_sum2(m.x, m.y);
      if ((threadIdx.x & 63) == 0) put(g, m);
    }
  }
}

// part: the moments of the pieces, few enough for every block to put its batch entry's together itself, a group a wave (null: the
// statistics are in `stat`).  (Those in LDS and those in memory are read in two ways: one pointer for both would have to be
// moved out of its LDS array for batch entries after the first.)
template <class T, int ACT, bool STREAM>
__global__ __launch_bounds__(1024) void norm_last_apply_kernel(NormArgs a, int active, const T* x, const float* gamma,
                                                               const float* beta, const Stat* stat, const double2* part, Cut cut,
                                                               float* mean, float* rstd, T* y) {
  constexpr int V = kVec<T>, U = 4;
  extern __shared__ double lds[];
  const int b = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  Stat* const mine = reinterpret_cast<Stat*>(lds);
  if (part != nullptr) {
    const bool tells = j == 0 && (threadIdx.x & 63) == 0;
    for (int g = threadIdx.x >> 6; g < a.G; g += blockDim.x >> 6) {
      const long long bg = (long long)b * a.G + g;
      const double2* const mine_of = part + bg * cut.pieces;
      double s = 0.0, q = 0.0;
      piece_share(cut, 0, mine_of, threadIdx.x & 63, 64, s, q);
      wave_sum2(s, q);
      const Stat st = stat_of(moments_of(mine_of[0].x, s * cut.inv, q * cut.inv), a.eps, tells ? mean : nullptr,
                              tells ? rstd : nullptr, bg);
      if ((threadIdx.x & 63) == 0) mine[g] = st;
    }
    __syncthreads();
  }
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
    store_any<STREAM>(y + at, repack(v));
  };
  sweep_last<V, U>(base, base + a.P * a.C, active, j, a.pieces, INT_MAX,
                   [&](long long at, long long step) {
                     pack<T> k[U];
#pragma unroll
                     for (int u = 0; u < U; ++u) k[u] = load_any<STREAM>(x + at + u * step);
#pragma unroll
                     for (int u = 0; u < U; ++u) put(at + u * step, k[u]);
                   },
                   [&](long long at) { put(at, load_any<STREAM>(x + at)); },
                   [&](long long at, int u) {
                     Affine g = f[0];
#pragma unroll
                     for (int w = 1; w < V; ++w)
                       if (w == u) g = f[w];
                     store1(y + at, normed<ACT>(g, load1(x + at)));
                   });
}

// part[(b, c)][piece] = (sum gz, sum gz xh)
template <class T, int ACT, bool STREAM>
__global__ __launch_bounds__(1024) void norm_last_grad_sum_kernel(NormArgs a, int active, const T* x, const T* gy,
                                                                  const float* gamma, const float* beta, const float* mean,
                                                                  const float* rstd, double2* part) {
  constexpr int V = kVec<T>, U = 2;
  extern __shared__ double2 pairs[];
  const int b = (int)blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  const long long base = (long long)b * a.P * a.C;
  Slope k[V];
  double s1[V], s2[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int c = ((int)threadIdx.x * V + u) % a.C;
    const long long bg = (long long)b * a.G + c / a.D;
    k[u] = slope_of<ACT>(mean[bg], rstd[bg], gamma ? gamma[c] : 1.f, beta ? beta[c] : 0.f);
    s1[u] = s2[u] = 0.0;
  }
  auto add1 = [&](int u, float v, float g) {
    float d, gz;
    terms<ACT>(k[u], v, g, d, gz);
    s1[u] += gz;
    s2[u] = fma((double)gz, (double)d, s2[u]);
  };
  auto add = [&](pack<T> px, pack<T> pg, float (&t1)[V], float (&t2)[V]) {
    float v[V], g[V];
    unpack(px, v);
    unpack(pg, g);
#pragma unroll
    for (int u = 0; u < V; ++u) {
      float d, gz;
      terms<ACT>(k[u], v[u], g[u], d, gz);
      t1[u] += gz;
      t2[u] = fmaf(gz, d, t2[u]);
    }
  };
  auto flush = [&](const float (&t1)[V], const float (&t2)[V]) {
#pragma unroll
    for (int u = 0; u < V; ++u) {
      s1[u] += t1[u];
      s2[u] += t2[u];
    }
  };
  sweep_last<V, U>(base, base + a.P * a.C, active, (long long)j * a.run, 1, a.run,
                   [&](long long at, long long step) {
                     pack<T> px[U], pg[U];
#pragma unroll
                     for (int u = 0; u < U; ++u) {
                       px[u] = load_any<STREAM>(x + at + u * step);
                       pg[u] = load_any<STREAM>(gy + at + u * step);
                     }
                     float t1[V] = {}, t2[V] = {};
#pragma unroll
                     for (int u = 0; u < U; ++u) add(px[u], pg[u], t1, t2);
                     flush(t1, t2);
                   },
                   [&](long long at) {
                     float t1[V] = {}, t2[V] = {};
                     add(load_any<STREAM>(x + at), load_any<STREAM>(gy + at), t1, t2);
                     flush(t1, t2);
                   },
                   [&](long long at, int u) {
                     const float v = load1(x + at), g = load1(gy + at);
#pragma unroll
                     for (int w = 0; w < V; ++w)
                       if (w == u) add1(w, v, g);
                   });
  if ((int)threadIdx.x < active) {
#pragma unroll
    for (int u = 0; u < V; ++u) pairs[threadIdx.x * V + u] = make_double2(s1[u], s2[u]);
  }
  const double2* const sums = channel_sums(pairs, active * V / a.C, a.C);
  for (int c = threadIdx.x; c < a.C; c += blockDim.x)
    part[((long long)b * a.C + c) * a.pieces + j] = make_double2(sums[c].x, sums[c].y * rstd[(long long)b * a.G + c / a.D]);
}

template <class T, int ACT, bool STREAM>
__global__ __launch_bounds__(1024) void norm_last_grad_apply_kernel(NormArgs a, unsigned mine, int active, const T* x, const T* gy,
                                                                    const float* gamma, const float* beta, const float* mean,
                                                                    const float* rstd, const float2* m, const double2* part, int parts,
                                                                    float* ggamma, float* gbeta, int accumulate, T* gx) {
  constexpr int V = kVec<T>, U = 2;
  extern __shared__ double lds[];
  if (blockIdx.x >= mine)
    return param_grads(a, parts, part, (long long)(blockIdx.x - mine) * (blockDim.x >> 6) + (threadIdx.x >> 6), ggamma, gbeta,
                       accumulate);
  const int b = blockIdx.x / a.pieces, j = blockIdx.x % a.pieces;
  float2* const own = reinterpret_cast<float2*>(lds);
  if (m == nullptr) {
    const long long b0 = (long long)b * a.G;
    for (int g = threadIdx.x >> 6; g < a.G; g += blockDim.x >> 6) {
      double s1 = 0.0, s2 = 0.0;
      group_share(a, parts, part, gamma, b0 + g, threadIdx.x & 63, 64, s1, s2);
      wave_sum2(s1, s2);
      if ((threadIdx.x & 63) == 0) own[g] = make_float2((float)(s1 * a.inv_n), (float)(s2 * a.inv_n));
    }
    __syncthreads();
  }
  const long long base = (long long)b * a.P * a.C;
  Slope k[V];
  Weights w[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const int c = ((int)threadIdx.x * V + u) % a.C, g = c / a.D;
    const float rs = rstd[(long long)b * a.G + g], ga = gamma ? gamma[c] : 1.f;
    k[u] = slope_of<ACT>(mean[(long long)b * a.G + g], rs, ga, beta ? beta[c] : 0.f);
    if (m == nullptr) w[u] = weights_of(rs, ga, own[g]);
    else w[u] = weights_of(rs, ga, m[(long long)b * a.G + g]);
  }
  auto put = [&](long long at, pack<T> px, pack<T> pg) {
    float v[V], g[V];
    unpack(px, v);
    unpack(pg, g);
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = grad_of<ACT>(k[u], w[u], v[u], g[u]);
    store_any<STREAM>(gx + at, repack(v));
  };
  sweep_last<V, U>(base, base + a.P * a.C, active, j, a.pieces, INT_MAX,
                   [&](long long at, long long step) {
                     pack<T> px[U], pg[U];
#pragma unroll
                     for (int u = 0; u < U; ++u) {
                       px[u] = load_any<STREAM>(x + at + u * step);
                       pg[u] = load_any<STREAM>(gy + at + u * step);
                     }
#pragma unroll
                     for (int u = 0; u < U; ++u) put(at + u * step, px[u], pg[u]);
                   },
                   [&](long long at) { put(at, load_any<STREAM>(x + at), load_any<STREAM>(gy + at)); },
                   [&](long long at, int u) {
                     const float v = load1(x + at), g = load1(gy + at);
#pragma unroll
                     for (int q = 0; q < V; ++q)
                       if (q == u) store1(gx + at, grad_of<ACT>(k[q], w[q], v, g));
                   });
}

// ------------------------------------------------------------------------------------------
// Groups that one block holds in its registers: one launch, x (and gy) read once.  A thread has 16 values of the group,
// those of whole 16-byte runs where the runs stay within a point's channels of the group (channels first: always), else
// every `threads`-th.  The adjoint's sums over a channel go through LDS.  Groups by batch entries in two dimensions of the grid: 2^23
// groups of 512 threads are more than one dimension holds.
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
      if (e + V <= s.n) q[k] = load_any<false>(x + small_at<LAST>(a, s, b, g, e));
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
        store_any<false>(y + small_at<LAST>(a, s, b, g, e), repack(w));
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
  const int b = blockIdx.y, g = blockIdx.x;
  float v[kSmallValues];
  small_load<T, LAST>(a, s, b, g, x, v);
  // k is the group's first value, whatever it is: differences and their squares are formed in double
  const double first = load1(x + small_at<LAST>(a, s, b, g, 0));
  double sum = 0.0, square = 0.0;
  small_values<T>(s, [&](int k, int) {
    const double d = v[k] - first;
    sum += d;
    square = fma(d, d, square);
  });
  block_sum2(sum, square, red);
  const bool tells = threadIdx.x == 0;
  const Stat st = stat_of(moments_of(first, sum * a.inv_n, square * a.inv_n), a.eps, tells ? mean : nullptr, tells ? rstd : nullptr,
                          (long long)b * a.G + g);
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
  const int b = blockIdx.y, g = blockIdx.x;
  const bool params = part != nullptr || ggamma != nullptr || gbeta != nullptr;
  float v[kSmallValues], w[kSmallValues];
  small_load<T, LAST>(a, s, b, g, x, v);
  small_load<T, LAST>(a, s, b, g, gy, w);
  for (int d = threadIdx.x; d < a.D; d += blockDim.x)
    affine[d] = make_float2(gamma ? gamma[g * a.D + d] : 1.f, beta ? beta[g * a.D + d] : 0.f);
  const long long bg = (long long)b * a.G + g;
  const float mu = mean[bg], rs = rstd[bg];
  float2* const product = reinterpret_cast<float2*>(lds);      // gz and gz xh of every value
  __syncthreads();
  double s1 = 0.0, s2 = 0.0;
  small_values<T>(s, [&](int k, int e) {                  // v: xh, w: gamma gz
    const float2 f = affine[small_channel<LAST>(a, s, e)];
    float d, gz;
    terms<ACT>(slope_of<ACT>(mu, rs, f.x, f.y), v[k], w[k], d, gz);
    v[k] = d * rs;
    w[k] = gz * f.x;
    s1 += w[k];
    s2 = fma((double)w[k], (double)v[k], s2);
    if (params) product[e] = make_float2(gz, gz * v[k]);
  });
  block_sum2(s1, s2, red);
  if (gx != nullptr) {
    const float m1 = (float)(s1 * a.inv_n), m2 = (float)(s2 * a.inv_n);
    small_values<T>(s, [&](int k, int) { w[k] = rs * ((w[k] - m1) - v[k] * m2); });
    small_store<T, LAST>(a, s, b, g, gx, w);
  }
  if (!params) return;
  // a channel's sums by `lanes` lanes or, where there are fewer channels than waves, by several waves
  const int nw = (int)blockDim.x >> 6, P = (int)a.P;
  auto put = [&](int d, double t1, double t2) {
    const int c = g * a.D + d;
    if (part != nullptr) part[(long long)b * a.C + c] = make_double2(t1, t2);
    else put_params(c, t1, t2, ggamma, gbeta, accumulate);
  };
  if (2 * a.D <= nw) {
    const int waves = nw / a.D, d = (int)(threadIdx.x >> 6) / waves, w = (int)(threadIdx.x >> 6) % waves;
    double t1 = 0.0, t2 = 0.0;
    if (d < a.D)
      for (int p = w * 64 + (threadIdx.x & 63); p < P; p += waves * 64) {
        const float2 q = product[LAST ? p * a.D + d : d * P + p];
        t1 += q.x;
        t2 += q.y;
      }
    wave_sum2(t1, t2);
    __syncthreads();                                      // (everybody has read what block_sum2 left in red)
    if ((threadIdx.x & 63) == 0) {
      red[2 * (threadIdx.x >> 6)] = t1;
      red[2 * (threadIdx.x >> 6) + 1] = t2;
    }
    __syncthreads();
    if ((int)threadIdx.x >= a.D) return;
    t1 = t2 = 0.0;
    for (int k = 0; k < waves; ++k) {
      t1 += red[2 * (threadIdx.x * waves + k)];
      t2 += red[2 * (threadIdx.x * waves + k) + 1];
    }
    put(threadIdx.x, t1, t2);
    return;
  }
  const int lane = threadIdx.x & (lanes - 1);
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
    if (d < a.D && lane == 0) put(d, t1, t2);
  }
}

// ------------------------------------------------------------------------------------------
// Launches
// ------------------------------------------------------------------------------------------
constexpr long long kSumBlocks = 4096;        // blocks of a launch that only reads: 16 a CU; channels last, half as many
constexpr long long kTileBytes = 16384;       // of a whole tile of 256 threads that read one field
constexpr long long kApplyBlocks = 1 << 22;   // of one that writes: a tile each, but for the very largest fields
// Where every block first adds the sums of pieces, fewer (adjoint of 24 rows of 357210: 512 blocks 35.0 us, 2048 33.6, a tile a block
// 35.0; of 20 rows of 700000 57.6, 56.0, 57.9), and channels last, where a thread first has its channels' factors to work out
// (5242880 points of 32 channels: 1024 blocks 340, 8192 327, a tile a block 332; bf16 adjoint, 2 x 4194304 points of 20: 341, 344, 488).
constexpr long long kApplyInside = 2048;
constexpr long long kApplyLast = 8192;
constexpr long long kShortRow = 512;          // rows below this go wave by wave: 4 x 64 rows of 600 take 8.7 us, 7.1 block by
                                              // block, 32 x 64 of them 9.8 and 10.2

NormArgs norm_args(const NormShape& n) {
  const int D = n.C / n.G;
  const double count = (double)n.P * D;
  return NormArgs{n.B, n.C, n.G, D, (long long)n.P, count > 0 ? 1.0 / count : 0.0, n.eps, 1, 1};
}

// Fields that the memory-side cache does not hold together are read and written with the nontemporal hint: the sums' launch
// 88 us without and 135 with the outputs of an earlier call that the cache still has to write back (60 x 60 x 64 x 30, 20
// channels).  Reading the second time from that cache, groups that fit it one after the other or backwards from where the sums
// ended, gained nothing: it gives 7 to 7.7 TB/s, the memory behind it 6.2.
bool streams(const NormShape& n, int fields) { return n.P * n.C * n.B * (n.bf16 ? 2 : 4) * (fields + 1) > kStreamBytes; }

// Threads of the channels-last kernels that take part: a multiple of what makes a step whole points.
int active_threads(int C, int V) {
  int g = C, h = V;
  while (h != 0) { const int r = g % h; g = h; h = r; }
  const int unit = C / g;
  return unit <= kThreads ? kThreads / unit * unit : unit;
}

// Deals the `tiles` tiles of each of `ranges` ranges to blocks, about `blocks` in all.
void deal(NormArgs& a, long long ranges, long long tiles, long long blocks) {
  long long p = (blocks + ranges - 1) / ranges;
  if (p > tiles) p = tiles;
  if (p < 1) p = 1;
  a.run = (int)((tiles + p - 1) / p);
  a.pieces = (int)(a.run > 0 ? (tiles + a.run - 1) / a.run : 1);
}
// values of a whole tile where `fields` fields are read
long long tile_values(const NormShape& n, int fields) { return kTileBytes / fields / (n.bf16 ? 2 : 4); }
NormArgs cut_groups(const NormShape& n) {              // channels first, statistics
  NormArgs a = norm_args(n);
  const long long tile = tile_values(n, 1);
  deal(a, (long long)n.B * n.G, (a.P * a.D + tile - 1) / tile, kSumBlocks);
  return a;
}
NormArgs cut_rows(const NormShape& n, int fields, long long blocks) {  // channels first, where channels count
  NormArgs a = norm_args(n);
  const long long tile = tile_values(n, fields);
  if (n.P >= kShortRow) deal(a, (long long)n.B * n.C, (n.P + tile - 1) / tile, blocks);
  return a;
}
// Channels last: blocks of at least 64 points, whose sums (16 bytes a channel) are then little beside them, and of at least
// three tiles where they only read (every piece is one more to add: 400000 points of 20 channels, forward with one tile 26.4 us, two
// 23.8, three 23.6, six 23.6; adjoint 40.6, 40.5, 38.3, 38.0), but no fewer than 256 in all (bf16, 4 x 13440 points of 27: 64 blocks
// 13.0, 128 12.5, 256 and more 12.3; adjoint of 20000 points of 256: 256 29.6, 1024 34.0).
NormArgs cut_points(const NormShape& n, int fields, long long blocks, int tiles_at_least) {
  NormArgs a = norm_args(n);
  const long long tile = (long long)active_threads(n.C, n.bf16 ? 8 : 4) * (n.bf16 ? 8 : 4) * (fields == 1 ? 4 : 2);
  const long long tiles = (n.P * n.C + tile - 1) / tile;
  long long most = n.B * (n.P / 64 + 1);
  if (most > n.B * tiles / tiles_at_least && n.B * tiles > 256) most = n.B * tiles / tiles_at_least;
  if (most < 256) most = 256;
  deal(a, n.B, tiles, blocks < most ? blocks : most);
  return a;
}

// The cuts of cut_groups() and, channels last, of cut_points(): piece j starts behind j stretches of whole tiles.
Cut cut_of(const NormShape& n, const NormArgs& a) {
  const long long range = n.last ? n.P * n.C : n.P * a.D;
  const int V = n.bf16 ? 8 : 4;
  const long long tile = n.last ? (long long)active_threads(n.C, V) * V * 4 : tile_values(n, 1);
  return Cut{range, a.run * tile, range > 0 ? 1.0 / (double)range : 0.0, a.pieces, n.last ? 1 : V};
}

// LDS of the channels-last sums: a pair for every value of the active threads, one more for every thread or channel
size_t pair_bytes(const NormShape& n, int active, int threads) {
  return ((size_t)active * (n.bf16 ? 8 : 4) + (threads > n.C ? threads : n.C)) * sizeof(double2);
}

// scratch: sums of pieces, statistics or means
size_t norm_part_bytes(const NormShape& n) {
  const NormArgs f = n.last ? cut_points(n, 1, kSumBlocks / 2, 3) : cut_groups(n);
  const NormArgs b = n.last ? cut_points(n, 2, kSumBlocks / 2, 3) : cut_rows(n, 2, kSumBlocks);
  const size_t fwd = (size_t)n.B * n.G * f.pieces, bwd = (size_t)n.B * n.C * b.pieces;
  return ((fwd > bwd ? fwd : bwd) * sizeof(double2) + 255) & ~size_t(255);
}

unsigned row_blocks(const NormArgs& a, bool short_rows) {
  const long long rows = (long long)a.B * a.C;
  return (unsigned)(short_rows ? (rows + kThreads / 64 - 1) / (kThreads / 64) : rows * a.pieces);
}

// Sums of pieces that every block of the next launch adds itself, sparing a launch: few of them, in small fields.  Us, this way
// and with the launch.  Channels first: adjoint of 20 x 80000 values, 800 sums, 12.7 and 13.4, of 20 x 200000, 1960 sums, 20.5 and
// 20.0, of 20 x 400000, 3920 sums, 36.0 and 33.9; fields of 32 MB 20.9 and 22.6, of 64 MB 38.7 and 41.2, of 128 MB 78.9 and 79.2,
// of 320 MB 172.8 and 160.7, as fewer and longer blocks write.  Channels last, where a block adds those of all its groups: 20
// channels in 4 groups, 400 sums 8.8 and 9.8, 800 sums 9.8 and 10.0; 64 in 16, 500 sums 10.4 and 9.7; 20 in 20, 1000 sums 11.1 and 9.7.
constexpr long long kInlineParts = 2048, kInlineBytes = 64ll << 20;
bool inline_parts(const NormShape& n, long long parts) {
  return parts <= (n.last ? kInlineParts / 4 : kInlineParts) && n.P * n.C * n.B * (n.bf16 ? 2 : 4) <= kInlineBytes;
}

// Whether one block takes a whole group.  Us, this way and in several launches: channels first, forward, 4 groups of 4096
// values 5.7 and 7.0, of 16000 7.3 and 7.7, 1024 of 8000 17 and 24.  Channels last, where a group is a narrow column of the
// field: 4 groups of 4096 7.3 and 8.1, of 16000 13.3 and 8.5, 512 groups of 512 (8 channels) 5.7 and 8.4, 512 of 4000 (2 channels)
// 25 and 12.
bool small_fits(const NormShape& n, bool adjoint) {
  const long long most = n.last ? (adjoint ? 2048 : 8192) : adjoint ? kSmallBwd : kSmallFwd;
  return n.P > 0 && n.P <= most && n.P * (n.C / n.G) <= most && (!n.last || n.P * n.C * n.B <= 1 << 19);
}
// blocks of norm_grad_fold_kernel for `count` groups or channels of `sums` sums each
unsigned fold_blocks(long long count, int sums) {
  const int each = fold_each(sums);
  return (unsigned)((count + each - 1) / each);
}
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

// f(std::integral_constant<bool, b>()...)
template <class F>
void with(bool b, F&& f) {
  if (b) f(std::true_type());
  else f(std::false_type());
}

// One launch after the other, none after one that was refused: the next one would read what that one had to leave.
struct Launches {
  hipError_t status = hipSuccess;
  template <class F>
  void operator()(F&& launch) {
    if (status != hipSuccess) return;
    launch();
    status = hipGetLastError();
  }
};

template <class T, int ACT>
hipError_t fwd(const NormShape& n, const T* x, const float* gamma, const float* beta, T* y, float* mean, float* rstd,
               void* ws, hipStream_t s) {
  double2* part = static_cast<double2*>(ws);
  Stat* stat = reinterpret_cast<Stat*>(static_cast<char*>(ws) + norm_part_bytes(n));
  if (small_fits(n, false)) {
    const NormArgs a = norm_args(n);
    const SmallArgs k = small_args(n, kVec<T>);
    with(n.last, [&](auto last) {
      hipLaunchKernelGGL((norm_small_kernel<T, ACT, decltype(last)::value>), dim3(n.G, n.B), dim3(small_threads(k.n)), 0, s, a, k, x,
                         gamma, beta, y, mean, rstd);
    });
    return hipGetLastError();
  }
  const bool hint = streams(n, 1);
  Launches then;
  if (n.last) {
    const NormArgs a = cut_points(n, 1, kSumBlocks / 2, 3), out = cut_points(n, 1, kApplyLast, 1);
    const int active = active_threads(n.C, kVec<T>), threads = (active + 63) / 64 * 64;
    const bool inside = n.P > 0 && inline_parts(n, (long long)n.G * a.pieces);
    const Cut cut = cut_of(n, a);
    const dim3 grid((unsigned)(n.B * a.pieces));
    with(hint, [&](auto stream) {
      constexpr bool S = decltype(stream)::value;
      then([&] {
        hipLaunchKernelGGL((norm_last_sum_kernel<T, S>), grid, dim3(threads), pair_bytes(n, active, threads), s, a, cut, active, x, part);
      });
      if (!inside) then([&] {
        hipLaunchKernelGGL(norm_stat_kernel, dim3(n.B * n.G), dim3(kThreads), 0, s, a, cut, part, stat, mean, rstd);
      });
      if (n.P > 0) then([&] {
        hipLaunchKernelGGL((norm_last_apply_kernel<T, ACT, S>), dim3((unsigned)(n.B * out.pieces)), dim3(threads),
                           inside ? n.G * sizeof(Stat) : 0, s, out, active, x, gamma, beta, stat, inside ? part : nullptr, cut, mean,
                           rstd, y);
      });
    });
    return then.status;
  }
  const NormArgs a = cut_groups(n);
  const Cut cut = cut_of(n, a);
  const bool short_rows = n.P < kShortRow, inside = !short_rows && inline_parts(n, a.pieces);
  const NormArgs rows = cut_rows(n, 1, inside ? kApplyInside : kApplyBlocks);
  with(hint, [&](auto stream) {
    constexpr bool S = decltype(stream)::value;
    then([&] {
      hipLaunchKernelGGL((norm_sum_kernel<T, S>), dim3((unsigned)(n.B * n.G * a.pieces)), dim3(kThreads), 0, s, a, cut, x, part);
    });
    if (!inside) then([&] {
      hipLaunchKernelGGL(norm_stat_kernel, dim3(n.B * n.G), dim3(kThreads), 0, s, a, cut, part, stat, mean, rstd);
    });
    with(short_rows, [&](auto short_) {
      then([&] {
        hipLaunchKernelGGL((norm_apply_kernel<T, ACT, decltype(short_)::value, S>), dim3(row_blocks(rows, short_rows)), dim3(kThreads), 0,
                           s, rows, x, gamma, beta, stat, inside ? part : nullptr, cut, mean, rstd, y);
      });
    });
  });
  return then.status;
}

template <class T, int ACT>
hipError_t bwd(const NormShape& n, const T* x, const float* gamma, const float* beta, const float* mean, const float* rstd,
               const T* gy, T* gx, float* ggamma, float* gbeta, int accumulate, void* ws, hipStream_t s) {
  double2* part = static_cast<double2*>(ws);
  float2* m = reinterpret_cast<float2*>(static_cast<char*>(ws) + norm_part_bytes(n));
  const bool params = ggamma != nullptr || gbeta != nullptr;
  Launches then;
  if (small_fits(n, true)) {
    const NormArgs a = norm_args(n);
    const SmallArgs k = small_args(n, kVec<T>);
    int lanes = 1;
    while (lanes < 64 && lanes < n.P) lanes *= 2;
    const bool later = params && n.B > 1;
    with(n.last, [&](auto last) {
      then([&] {
        hipLaunchKernelGGL((norm_small_grad_kernel<T, ACT, decltype(last)::value>), dim3(n.G, n.B), dim3(small_threads(k.n)),
                           params ? k.n * sizeof(float2) : 0, s, a, k, lanes, x, gy, gamma, beta, mean, rstd, gx, later ? part : nullptr,
                           ggamma, gbeta, accumulate);
      });
    });
    if (later) then([&] {
      hipLaunchKernelGGL(norm_grad_fold_kernel, dim3(fold_blocks(n.C, n.B * a.pieces)), dim3(kFoldThreads), 0, s, a, 0u, part, gamma, m,
                         ggamma, gbeta, accumulate);
    });
    return then.status;
  }
  const bool short_rows = !n.last && n.P < kShortRow, writes = gx != nullptr && n.P > 0;
  const NormArgs a = n.last ? cut_points(n, 2, kSumBlocks / 2, 3) : cut_rows(n, 2, kSumBlocks);
  const int active = active_threads(n.C, kVec<T>), threads = n.last ? (active + 63) / 64 * 64 : kThreads;
  const bool inside = writes && !short_rows && inline_parts(n, (long long)(n.last ? n.C : n.C / n.G) * a.pieces);
  const NormArgs out = n.last ? cut_points(n, 2, kApplyLast, 1) : cut_rows(n, 2, inside ? kApplyInside : kApplyBlocks);
  const unsigned channel_blocks = params ? (unsigned)((n.C + threads / 64 - 1) / (threads / 64)) : 0;
  const unsigned groups = fold_blocks((long long)n.B * n.G, a.D * a.pieces);
  const unsigned blocks = n.last ? (unsigned)(n.B * a.pieces) : row_blocks(a, short_rows);
  const unsigned own = n.last ? (unsigned)(n.B * out.pieces) : row_blocks(out, short_rows);
  const dim3 grid(own + (inside ? channel_blocks : 0));
  const float2* means = inside ? nullptr : m;
  auto fold = [&] {
    if (!inside) then([&] {
      hipLaunchKernelGGL(norm_grad_fold_kernel, dim3(groups + (params ? fold_blocks(n.C, n.B * a.pieces) : 0)), dim3(kFoldThreads), 0, s,
                         a, groups, part, gamma, m, ggamma, gbeta, accumulate);
    });
  };
  with(streams(n, 2), [&](auto stream) {
    constexpr bool S = decltype(stream)::value;
    if (n.last) {
      then([&] {
        hipLaunchKernelGGL((norm_last_grad_sum_kernel<T, ACT, S>), dim3(blocks), dim3(threads), pair_bytes(n, active, threads), s, a,
                           active, x, gy, gamma, beta, mean, rstd, part);
      });
      fold();
      if (writes) then([&] {
        hipLaunchKernelGGL((norm_last_grad_apply_kernel<T, ACT, S>), grid, dim3(threads), inside ? n.G * sizeof(float2) : 0, s, out, own,
                           active, x, gy, gamma, beta, mean, rstd, means, part, a.pieces, ggamma, gbeta, accumulate, gx);
      });
      return;
    }
    with(short_rows, [&](auto short_) {
      constexpr bool R = decltype(short_)::value;
      then([&] {
        hipLaunchKernelGGL((norm_grad_sum_kernel<T, ACT, R, S>), dim3(blocks), dim3(kThreads), 0, s, a, x, gy, gamma, beta, mean, rstd,
                           part);
      });
      fold();
      if (writes) then([&] {
        hipLaunchKernelGGL((norm_grad_apply_kernel<T, ACT, R, S>), grid, dim3(kThreads), 0, s, out, own, x, gy, gamma, beta, mean, rstd,
                           means, part, a.pieces, ggamma, gbeta, accumulate, gx);
      });
    });
  });
  return then.status;
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
