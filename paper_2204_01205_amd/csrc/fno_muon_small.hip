// The Muon step of small real matrices (the lift's, the blocks', the projection's): a block has one, X and its Gram matrix stay in
// LDS.  A network has a handful of them, of a few thousand values: what counts is the latency of five iterations of three dependent
// products, so a thread takes single entries, and the sums over the longer side are split where there are more threads than entries.
#include "fno_muon.h"

namespace fno {

namespace {

constexpr int kSmallThreads = 512;
constexpr int kPerLaunch = 48;         // tensors whose addresses go with one launch's arguments

struct SmallEntry {
  float* p;
  const float* g;
  float* mom;
  unsigned first;                      // first matrix of the launch that belongs to this tensor
  unsigned skip;                       // matrices of it in earlier launches
  int rows, cols;
  float keep, move;                    // 1 - lr weight_decay, lr scale
};
struct SmallList {
  SmallEntry t[kPerLaunch];
  int count;
};

// e / n and e % n for e n < 2^32
struct Divisor {
  unsigned n, inv;
  __device__ explicit Divisor(unsigned n) : n(n), inv(n == 1 ? 0u : 0xFFFFFFFFu / n + 1u) {}
  __device__ __forceinline__ void split(unsigned e, unsigned& q, unsigned& r) const {
    q = n == 1 ? e : __umulhi(e, inv);
    r = e - q * n;
  }
};

__global__ __launch_bounds__(kSmallThreads) void muon_small_kernel(SmallList l, MuonScalars c) {
  extern __shared__ float mem[];
  __shared__ double red[kSmallThreads / 64];
  float scale;
  if (!muon_scale(c, scale)) return;
  int k = 0;
  while (k + 1 < l.count && l.t[k + 1].first <= blockIdx.x) ++k;
  const SmallEntry& t = l.t[k];
  const bool tall = t.rows > t.cols;
  const unsigned m = tall ? t.cols : t.rows, n = tall ? t.rows : t.cols, mn = m * n, mm = m * m, tid = threadIdx.x;
  const unsigned xs = n | 1, as = m | 1;           // odd strides: a column spreads over the banks
  float *x = mem, *y = x + m * xs, *const A = y + m * xs, *const Q = A + m * as, *const part = Q + m * as;
  const long long base = ((long long)(blockIdx.x - t.first) + t.skip) * mn;
  const Divisor by_cols(t.cols), by_n(n), by_m(m);

  double sum = 0.0;
  for (unsigned e = tid; e < mn; e += kSmallThreads) {
    unsigned i, j;
    by_cols.split(e, i, j);
    float mo = t.mom[base + e];
    const float u = muon_momentum(c, t.g[base + e] * scale, mo);
    t.mom[base + e] = mo;
    x[tall ? j * xs + i : i * xs + j] = u;
    sum = fma((double)u, (double)u, sum);
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
  if ((tid & 63) == 0) red[tid >> 6] = sum;
  __syncthreads();
  sum = 0.0;
  for (int w = 0; w < kSmallThreads / 64; ++w) sum += red[w];
  const double inv = muon_inverse(sum, c.eps);
  for (unsigned e = tid; e < mn; e += kSmallThreads) {
    unsigned i, j;
    by_n.split(e, i, j);
    x[i * xs + j] = (float)(x[i * xs + j] * inv);
  }
  __syncthreads();

  unsigned parts = 1;                              // of the sums over n
  while (parts < 64 && 2 * parts * mm <= kSmallThreads && 8 * parts <= n) parts *= 2;
  const unsigned share = (n + parts - 1) / parts;
  for (int it = 0; it < c.iterations; ++it) {
    for (unsigned e = tid; e < mm * parts; e += kSmallThreads) {
      unsigned f = e, h = 0, i, j;
      while (f >= mm) {
        f -= mm;
        ++h;
      }
      by_m.split(f, i, j);
      const unsigned end = (h + 1) * share < n ? (h + 1) * share : n;
      const float *a = x + i * xs, *b = x + j * xs;
      float s0 = 0.f, s1 = 0.f;
      unsigned q = h * share;
      for (; q + 4 <= end; q += 4) {
        s0 = fmaf(a[q], b[q], s0);
        s1 = fmaf(a[q + 1], b[q + 1], s1);
        s0 = fmaf(a[q + 2], b[q + 2], s0);
        s1 = fmaf(a[q + 3], b[q + 3], s1);
      }
      for (; q < end; ++q) s0 = fmaf(a[q], b[q], s0);
      (parts == 1 ? A[i * as + j] : part[e]) = s0 + s1;
    }
    __syncthreads();
    if (parts > 1) {
      for (unsigned e = tid; e < mm; e += kSmallThreads) {
        unsigned i, j;
        by_m.split(e, i, j);
        float s = part[e];
        for (unsigned h = 1; h < parts; ++h) s += part[h * mm + e];
        A[i * as + j] = s;
      }
      __syncthreads();
    }
    for (unsigned e = tid; e < mm; e += kSmallThreads) {
      unsigned i, j;
      by_m.split(e, i, j);
      float s0 = 0.f, s1 = 0.f;
      unsigned q = 0;
      for (; q + 2 <= m; q += 2) {                 // A is symmetric: row j for column j
        s0 = fmaf(A[i * as + q], A[j * as + q], s0);
        s1 = fmaf(A[i * as + q + 1], A[j * as + q + 1], s1);
      }
      if (q < m) s0 = fmaf(A[i * as + q], A[j * as + q], s0);
      Q[i * as + j] = fmaf(c.b, A[i * as + j], c.c * (s0 + s1));
    }
    __syncthreads();
    for (unsigned e = tid; e < mn; e += kSmallThreads) {
      unsigned i, j;
      by_n.split(e, i, j);
      float s0 = c.a * x[i * xs + j], s1 = 0.f;
      unsigned q = 0;
      for (; q + 2 <= m; q += 2) {
        s0 = fmaf(Q[i * as + q], x[q * xs + j], s0);
        s1 = fmaf(Q[i * as + q + 1], x[(q + 1) * xs + j], s1);
      }
      if (q < m) s0 = fmaf(Q[i * as + q], x[q * xs + j], s0);
      y[i * xs + j] = s0 + s1;
    }
    __syncthreads();
    float* const z = x;
    x = y;
    y = z;
  }
  for (unsigned e = tid; e < mn; e += kSmallThreads) {
    unsigned i, j;
    by_cols.split(e, i, j);
    t.p[base + e] = fmaf(t.p[base + e], t.keep, -t.move * x[tall ? j * xs + i : i * xs + j]);
  }
}

size_t small_bytes(int m, int n) {
  return ((size_t)2 * m * (n | 1) + 2 * m * (m | 1) + kSmallThreads) * sizeof(float);
}

}  // namespace

bool muon_is_small(const MuonTensor& t) {
  const int m = t.rows < t.cols ? t.rows : t.cols;
  return !t.modes && m <= 32 && (long long)t.rows * t.cols <= 8192;
}

// Stacks go in launches of 2^22 matrices at most.
hipError_t launch_muon_small(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s) {
  constexpr long long kMost = 1ll << 22;
  SmallList l;
  l.count = 0;
  long long blocks = 0;
  size_t bytes = 0;
  auto flush = [&]() {
    hipError_t e = hipSuccess;
    if (l.count > 0) {
      e = ask_local_memory(reinterpret_cast<const void*>(muon_small_kernel), bytes + kSmallThreads / 64 * sizeof(double));
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(muon_small_kernel, dim3((unsigned)blocks), dim3(kSmallThreads), bytes, s, l, c);
      e = hipGetLastError();
    }
    l.count = 0;
    blocks = 0;
    bytes = 0;
    return e;
  };
  for (int k = 0; k < count; ++k) {
    if (!muon_is_small(t[k])) continue;
    for (long long done = 0; done < t[k].batch;) {
      if (l.count == kPerLaunch || blocks == kMost) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
      }
      const long long here = t[k].batch - done < kMost - blocks ? t[k].batch - done : kMost - blocks;
      l.t[l.count++] = SmallEntry{t[k].p, t[k].g, t[k].m, (unsigned)blocks, (unsigned)done, t[k].rows, t[k].cols,
                                  (float)(1.0 - lr * t[k].decay), (float)(lr * t[k].scale)};
      const int m = t[k].rows < t[k].cols ? t[k].rows : t[k].cols;
      const size_t need = small_bytes(m, t[k].rows + t[k].cols - m);
      bytes = need > bytes ? need : bytes;
      blocks += here;
      done += here;
    }
  }
  return flush();
}

}  // namespace fno
