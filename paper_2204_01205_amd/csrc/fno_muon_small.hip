// The Muon step of small real matrices (the lift's, the blocks', the projection's): a block has one.
//
// A network has a handful of them, of a few thousand values: what counts is the latency of five iterations of three dependent
// products.  X, m x n with m <= n, stays in LDS; its columns go in tiles of 16, which the block's waves own.  With 16 x 16 tiles of
// v_mfma_f32_16x16x4, whose lane (c, g) = (lane % 16, lane / 16) holds rows 4 g + r of column c of a result:
//   A = X X^T: a wave adds up its own columns', and the sums of all waves go through LDS: one barrier an iteration;
//   B = a + b A + c A A, by every wave for itself, and X = B X, its own columns': with the steps of a product taken in the order 4 g + r the
//   registers of a result are the operands of the next one, A and B being symmetric.
// 8 x 8 takes 0.5 us an iteration, 32 x 32 1.7, 32 x 256 4.1 (a thread for every entry of a product: 1.0, 5.0 and 24).
// Short wide matrices are folded: with m <= 8 (4) two (four) stretches of columns lie one below the other, and the blocks on the
// diagonal of their Gram matrix add up to A.
#include "fno_muon.h"

#include <algorithm>

namespace fno {

namespace {

constexpr int kWaves = 4, kMostWaves = 8;          // that own columns; of a block
constexpr int kPerLaunch = 48;         // tensors whose addresses go with one launch's arguments

// How a matrix lies in LDS: 2^lg rows a stretch of columns, of which m are there, `each` columns of `pitch` places.
struct SmallLayout {
  int m, n, lg, each, pitch, tiles;
  SmallLayout(int rows, int cols) {
    m = rows < cols ? rows : cols;
    n = rows < cols ? cols : rows;
    lg = m > 16 ? 5 : 4;
    while (lg > 2 && m <= 1 << (lg - 1) && lg < 5 && n > (16 * kWaves << (4 - lg))) --lg;
    const int folds = lg < 4 ? 16 >> lg : 1;
    each = (n + folds - 1) / folds;
    tiles = (each + 15) / 16;
    // 20 more than a multiple of 64: 16 rows by 4 columns of a tile lie in 64 banks, and so do 4 rows four apart by 16 columns
    pitch = (16 * tiles + 43) / 64 * 64 + 20;
  }
  int waves() const { return tiles < kWaves ? tiles : kWaves; }
  // up to eight waves for the memory's sake: 32 x 256 takes 12 us for its loads and stores alone with four
  int block_waves() const { return std::max(waves(), std::min(kMostWaves, (m * n + 255) / 256)); }
  size_t values() const { return (size_t)m * (lg < 4 ? 16 >> lg : 1) * pitch; }
  size_t sums() const { return (size_t)2 * waves() * (lg == 5 ? 4 : 1) * 256; }
};

struct SmallEntry {
  float* p;
  const float* g;
  float* mom;
  unsigned first;                      // first matrix of the launch that belongs to this tensor
  unsigned skip;                       // matrices of it in earlier launches
  int rows, cols, lg, each, pitch;
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

__device__ __forceinline__ v4f mfma16(float a, float b, v4f c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }
constexpr int kBatch = 8;              // values of a thread on their way at a time

// The iterations, T = 1 or 2 tiles of 16 rows.  sums: [2][waves][T][T][64 lanes], which take turns.
template <int T>
__device__ __forceinline__ void iterate(const MuonScalars& c, const SmallEntry& t, int m, float* x, v4f* sums) {
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, g = lane >> 4;
  const int tiles = (t.each + 15) / 16, waves = tiles < kWaves ? tiles : kWaves, side = (1 << t.lg) - 1;
  // rows that are not there are read as the last one of their stretch; what they make of A is cleared
  auto place = [&](int v) {
    const int i = v & side;
    return ((v >> t.lg) * m + (i < m ? i : m - 1)) * t.pitch;
  };
  int rows[T], cols[T][4];
  bool in[T][4];
#pragma unroll
  for (int I = 0; I < T; ++I) {
    rows[I] = place(16 * I + col) + g;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      cols[I][r] = place(16 * I + 4 * g + r) + col;
      in[I][r] = ((16 * I + 4 * g + r) & side) < m;
    }
  }
  for (int it = 0; it < c.iterations; ++it) {
    v4f* const mine = sums + (it & 1) * (waves * T * T * 64);
    v4f a[T][T];
#pragma unroll
    for (int I = 0; I < T; ++I)
#pragma unroll
      for (int K = 0; K < T; ++K) a[I][K] = v4f{0.f, 0.f, 0.f, 0.f};
    if (w < waves) {
      for (int J = w; J < tiles; J += kWaves) {
        float v[4][T];
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int I = 0; I < T; ++I) v[n][I] = x[rows[I] + 16 * J + 4 * n];
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int I = 0; I < T; ++I)
#pragma unroll
            for (int K = 0; K < T; ++K) a[I][K] = mfma16(v[n][I], v[n][K], a[I][K]);
      }
#pragma unroll
      for (int I = 0; I < T; ++I)
#pragma unroll
        for (int K = 0; K < T; ++K) mine[((w * T + I) * T + K) * 64 + lane] = a[I][K];
    }
    __syncthreads();
    if (w >= waves) continue;
#pragma unroll
    for (int I = 0; I < T; ++I)
#pragma unroll
      for (int K = 0; K < T; ++K) {
        v4f s = mine[(I * T + K) * 64 + lane];
        for (int v = 1; v < waves; ++v) s += mine[((v * T + I) * T + K) * 64 + lane];
        if (T == 1 && t.lg < 4) {
#pragma unroll
          for (int r = 0; r < 4; ++r) s[r] = (4 * g + r) >> t.lg == col >> t.lg ? s[r] : 0.f;
#pragma unroll
          for (int r = 0; r < 4; ++r) s[r] += __shfl_xor(s[r], 40);
          if (t.lg == 2)
#pragma unroll
            for (int r = 0; r < 4; ++r) s[r] += __shfl_xor(s[r], 20);
#pragma unroll
          for (int r = 0; r < 4; ++r) s[r] = (4 * g + r) >> t.lg == col >> t.lg ? s[r] : 0.f;
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) a[I][K][r] = in[I][r] && ((16 * K + col) & side) < m ? s[r] : 0.f;
      }
    v4f q[T][T];
#pragma unroll
    for (int I = 0; I < T; ++I)
#pragma unroll
      for (int K = 0; K < T; ++K) {
        v4f s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int L = 0; L < T; ++L)
#pragma unroll
          for (int r = 0; r < 4; ++r) s = mfma16(a[L][I][r], a[L][K][r], s);
#pragma unroll
        for (int r = 0; r < 4; ++r) q[I][K][r] = fmaf(c.b, a[I][K][r], c.c * s[r]) + (I == K && 4 * g + r == col ? c.a : 0.f);
      }
    for (int J = w; J < tiles; J += kWaves) {
      float v[T][4];
      v4f s[T];
#pragma unroll
      for (int L = 0; L < T; ++L)
#pragma unroll
        for (int r = 0; r < 4; ++r) v[L][r] = x[cols[L][r] + 16 * J];
#pragma unroll
      for (int I = 0; I < T; ++I) {
        s[I] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int L = 0; L < T; ++L)
#pragma unroll
          for (int r = 0; r < 4; ++r) s[I] = mfma16(q[L][I][r], v[L][r], s[I]);
      }
#pragma unroll
      for (int I = 0; I < T; ++I)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (in[I][r]) x[cols[I][r] + 16 * J] = s[I][r];
    }
    // the wave's own stores, before its loads of the next iteration, in the order of the program
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_wave_barrier();
  }
}

__global__ __launch_bounds__(64 * kMostWaves) void muon_small_kernel(SmallList l, MuonScalars c) {
  extern __shared__ __align__(16) float mem[];
  __shared__ double red[kMostWaves];
  float scale;
  if (!muon_scale(c, scale)) return;
  int k = 0;
  while (k + 1 < l.count && l.t[k + 1].first <= blockIdx.x) ++k;
  const SmallEntry& t = l.t[k];
  const bool tall = t.rows > t.cols;
  const unsigned m = tall ? t.cols : t.rows, mn = t.rows * t.cols, tid = threadIdx.x, threads = blockDim.x;
  const unsigned folds = t.lg < 4 ? 16 >> t.lg : 1, tiles = (t.each + 15) / 16, waves = tiles < kWaves ? tiles : kWaves;
  const unsigned each_sums = t.lg == 5 ? 4 * 64 : 64;
  v4f* const sums = reinterpret_cast<v4f*>(mem);
  float* const x = mem + 2 * waves * each_sums * 4;
  const long long base = ((long long)(blockIdx.x - t.first) + t.skip) * mn;
  const Divisor by_cols(t.cols), by_each(t.each);
  auto place = [&](unsigned e) {
    unsigned i, j, f, p;
    by_cols.split(e, i, j);
    by_each.split(tall ? i : j, f, p);
    return (f * m + (tall ? j : i)) * t.pitch + p;
  };

  for (unsigned e = tid; e < m * folds * t.pitch; e += threads) x[e] = 0.f;
  __syncthreads();
  double sum = 0.0;
  for (unsigned e0 = tid; e0 < mn; e0 += kBatch * threads) {
    float u[kBatch], mo[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const unsigned e = e0 + b * threads < mn ? e0 + b * threads : e0;
      u[b] = t.g[base + e];
      mo[b] = t.mom[base + e];
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const unsigned e = e0 + b * threads;
      if (e >= mn) continue;
      u[b] = muon_momentum(c, u[b] * scale, mo[b]);
      t.mom[base + e] = mo[b];
      x[place(e)] = u[b];
      sum = fma((double)u[b], (double)u[b], sum);
    }
  }
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) sum += __shfl_xor(sum, off);
  if ((tid & 63) == 0) red[tid >> 6] = sum;
  __syncthreads();
  sum = 0.0;
  for (unsigned w = 0; w < threads / 64; ++w) sum += red[w];
  const double inv = muon_inverse(sum, c.eps);
  for (unsigned e = tid; e < m * folds * t.pitch; e += threads) x[e] = (float)(x[e] * inv);
  __syncthreads();

  if (t.lg == 5) iterate<2>(c, t, (int)m, x, sums);
  else iterate<1>(c, t, (int)m, x, sums);
  __syncthreads();
  for (unsigned e0 = tid; e0 < mn; e0 += kBatch * threads) {
    float p[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) p[b] = t.p[base + (e0 + b * threads < mn ? e0 + b * threads : e0)];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const unsigned e = e0 + b * threads;
      if (e < mn) t.p[base + e] = fmaf(p[b], t.keep, -t.move * x[place(e)]);
    }
  }
}

}  // namespace

// A block's LDS at most: 16384 values; in each of 32 rows up to 3 more for the folds and 67 of padding; 8192 of sums.
constexpr int kMostValues = 16384;
constexpr size_t kMostLocal = (kMostValues + 32 * (3 + 67) + 8192) * sizeof(float);

// What fits a block's LDS.  us a step of one matrix, here and tile by tile (fno_muon_dense.hip): 8 x 8 8 and 60, 32 x 256 30 and 73, 32
// x 512 49 and 84; of 1024 of 32 x 512 210 and 835.
bool muon_is_small(const MuonTensor& t) {
  const int m = t.rows < t.cols ? t.rows : t.cols;
  return !t.modes && m <= 32 && (long long)t.rows * t.cols <= kMostValues;
}

// Stacks go in launches of 2^22 matrices at most.
hipError_t launch_muon_small(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s) {
  constexpr long long kMost = 1ll << 22;
  SmallList l;
  l.count = 0;
  long long blocks = 0;
  size_t bytes = 0;
  int waves = 0;
  auto flush = [&]() {
    hipError_t e = hipSuccess;
    if (l.count > 0) {
      e = ask_local_memory(reinterpret_cast<const void*>(muon_small_kernel), bytes, kMostLocal);
      if (e != hipSuccess) return e;
      hipLaunchKernelGGL(muon_small_kernel, dim3((unsigned)blocks), dim3(64 * waves), bytes, s, l, c);
      e = hipGetLastError();
    }
    l.count = 0;
    blocks = 0;
    bytes = 0;
    waves = 0;
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
      const SmallLayout y(t[k].rows, t[k].cols);
      l.t[l.count++] = SmallEntry{t[k].p, t[k].g, t[k].m, (unsigned)blocks, (unsigned)done, t[k].rows, t[k].cols, y.lg, y.each, y.pitch,
                                  (float)(1.0 - lr * t[k].decay), (float)(lr * t[k].scale)};
      const size_t need = (y.values() + y.sums()) * sizeof(float);
      bytes = need > bytes ? need : bytes;
      waves = std::max(waves, y.block_waves());
      blocks += here;
      done += here;
    }
  }
  return flush();
}

}  // namespace fno
