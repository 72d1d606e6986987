// The Muon step of larger real matrices: X, m x n with m <= n, kept in scratch.
//
// Of the three products of an iteration the first two, A = X X^T and B = b A + c A A, are symmetric and half of their tiles are
// worked out; the third is X = a X + B X.  They run on 16-bit matrix instructions: a value is the sum of two fp16 ones (the
// second holds what the first rounds off, together 22 bits), and of the four products of two such pairs three count.  That is a third of
// the 16-bit rate, five times the rate of single-precision products.  X, A and B are scaled by powers of two (kX, kA, kB) so that values
// up to 64, 256 and 1024 fit; what the pairs cannot hold, half of fp16's smallest step, is then 2^-35, 2^-33 and 2^-31.  For values from 2^-13,
// 2^-11 and 2^-9 on the 22 bits are the limit.
//
// All operands are read along their inner dimension: X by rows and by columns (both are written), A and B are symmetric.  A row
// is stored in pieces of 32 values, 64 bytes of first parts and 64 of second parts, a cache line that goes to LDS as it is; the
// 16-byte pieces of a row are permuted by the row, so that the 16 rows that a phase of an LDS read takes lie in different banks.
//
// Five iterations of 4 x 1024 x 1024, 1024 x 4096, 4096 x 1024 and 1000 x 1536 (254 GFLOP) take 1.23 ms: 620 TFLOP/s of 16-bit
// products, where a product of 8192^3 by the library reaches 1070; X = a X + B X alone runs at 770, the symmetric products, with fewer
// tiles than fit the chip twice, at 590.  A step of 32 of a tile of 128 reads 64 KB of LDS and writes 32 for some 768 cycles of matrix
// instructions, 125 bytes a cycle, which is about what LDS gives.  Smaller matrices are bound by their launches, three or four of 7 to 9 us an iteration (256 x
// 256).
//
// All matrices of a list go through a launch together, tile by tile.  Where these are too few for the chip, the sums are split over
// blocks and added by a launch of their own.
#include "fno_muon.h"

namespace fno {

namespace {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef _Float16 half;

constexpr float kX = 1024.f, kA = 256.f, kB = 64.f;
constexpr int kPerLaunch = 16;         // matrices or stacks whose addresses go with one launch's arguments
constexpr int kPieces = 256;           // partial sums of a matrix's norm, at most
constexpr int kPieceValues = 16 * kThreads;
constexpr int kStep = 32;              // inner dimension that goes to LDS at a time

struct DenseEntry {
  float* p;
  const float* g;
  float* mom;
  char* ws;                            // of the first matrix; each has `region` bytes
  long long part_at[3];                // split sums of the products, [matrix][split][tile], from the list's
  long long region, run;               // run: values of a piece of the norm
  int rows, cols, m, n, mp, np;        // mp, np: m and n up to whole tiles
  unsigned count, pieces;
  unsigned first_piece, first_tile;    // blocks of earlier entries: momentum, parts
  unsigned first[3], splits[3];        // and of the three products; blocks that share a tile's sum
  unsigned first_sum[3];               // tiles of earlier entries, where sums are split
  float keep, move;
};
struct DenseList {
  DenseEntry t[kPerLaunch];
  float* part;
  int count;
};

// Places of a matrix's arrays in its region
struct Region {
  half *x, *xt, *a, *b;
  long long next;                      // from one of the two arrays by columns to the other
  double* norm;
};
__host__ __device__ __forceinline__ long long region_bytes(long long mp, long long np) {
  return 12 * mp * np + 8 * mp * mp + kPieces * (long long)sizeof(double);
}
__device__ __forceinline__ Region region_of(const DenseEntry& t, unsigned matrix) {
  Region r;
  char* at = t.ws + matrix * t.region;
  const long long mn = 4ll * t.mp * t.np, mm = 4ll * t.mp * t.mp;
  r.x = reinterpret_cast<half*>(at);
  r.xt = reinterpret_cast<half*>(at + mn);
  r.next = mn / 2;
  r.a = reinterpret_cast<half*>(at + 3 * mn);
  r.b = reinterpret_cast<half*>(at + 3 * mn + mm);
  r.norm = reinterpret_cast<double*>(at + 3 * mn + 2 * mm);
  return r;
}
// The first part of value k of a row, rows of ld values; the second part lies 32 further on.
__device__ __forceinline__ long long pair_at(long long row, int ld, int k) { return row * 2 * ld + (k >> 5) * 64 + (k & 31); }

template <class F>
__device__ __forceinline__ const DenseEntry& entry_of(const DenseList& l, F&& first) {
  int k = 0;
  while (k + 1 < l.count && first(l.t[k + 1]) <= blockIdx.x) ++k;
  return l.t[k];
}

__device__ __forceinline__ double dense_block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kThreads) void dense_momentum_kernel(DenseList l, MuonScalars c) {
  __shared__ double red[kThreads / 64];
  float scale;
  if (!muon_scale(c, scale)) return;
  const DenseEntry& t = entry_of(l, [](const DenseEntry& e) { return e.first_piece; });
  const unsigned local = blockIdx.x - t.first_piece, matrix = local / t.pieces, piece = local % t.pieces;
  const long long values = (long long)t.rows * t.cols, begin = piece * t.run;
  const long long end = begin + t.run < values ? begin + t.run : values;
  const float* const g = t.g + matrix * values;
  float* const mom = t.mom + matrix * values;
  double sum = 0.0;
  long long at = begin;
  for (; at + kPieceValues <= end; at += kPieceValues) {
    typedef v4f loose __attribute__((aligned(4)));
    v4f u[4], mo[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u[q] = *reinterpret_cast<const loose*>(g + at + (q * kThreads + threadIdx.x) * 4);
      mo[q] = *reinterpret_cast<const loose*>(mom + at + (q * kThreads + threadIdx.x) * 4);
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float m = mo[q][k];
        const float v = muon_momentum(c, u[q][k] * scale, m);
        mo[q][k] = m;
        sum = fma((double)v, (double)v, sum);
      }
      *reinterpret_cast<loose*>(mom + at + (q * kThreads + threadIdx.x) * 4) = mo[q];
    }
  }
  for (long long i = at + threadIdx.x; i < end; i += kThreads) {
    float mo = mom[i];
    const float u = muon_momentum(c, g[i] * scale, mo);
    mom[i] = mo;
    sum = fma((double)u, (double)u, sum);
  }
  sum = dense_block_sum(sum, red);
  if (threadIdx.x == 0) region_of(t, matrix).norm[piece] = sum;
}

// X by rows and by columns as pairs, a 64 x 64 tile a block; without iterations the step itself.
__global__ __launch_bounds__(kThreads) void dense_parts_kernel(DenseList l, MuonScalars c) {
  __shared__ double red[kThreads / 64];
  __shared__ float tile[64][65];
  float scale;
  if (!muon_scale(c, scale)) return;
  const DenseEntry& t = entry_of(l, [](const DenseEntry& e) { return e.first_tile; });
  const unsigned tn = t.np / 64, tiles = t.mp / 64 * tn, local = blockIdx.x - t.first_tile, matrix = local / tiles;
  const int i0 = (int)(local % tiles / tn) * 64, j0 = (int)(local % tiles % tn) * 64;
  const Region r = region_of(t, matrix);
  const int tid = threadIdx.x;
  const double inv = muon_inverse(dense_block_sum(tid < (int)t.pieces ? r.norm[tid] : 0.0, red), c.eps);
  const bool tall = t.rows > t.cols;
  const int r0 = tall ? j0 : i0, c0 = tall ? i0 : j0, cc = c0 + (tid & 63);
  const long long base = (long long)matrix * t.rows * t.cols;
#pragma unroll 4
  for (int q = tid >> 6; q < 64; q += 4) {
    const bool here = r0 + q < t.rows && cc < t.cols;
    const long long at = base + (long long)(here ? r0 + q : 0) * t.cols + (here ? cc : 0);
    const float mo = t.mom[at], u = c.nesterov ? fmaf(c.mu, mo, t.g[at] * scale) : mo;
    const float v = here ? (float)(u * inv) : 0.f;
    if (c.iterations == 0) {
      if (here) t.p[at] = fmaf(t.p[at], t.keep, -t.move * v);
    } else {
      tile[tall ? tid & 63 : q][tall ? q : tid & 63] = v * kX;
    }
  }
  if (c.iterations == 0) return;
  __syncthreads();
#pragma unroll
  for (int q = tid; q < 512; q += kThreads) {
    const int line = q >> 3, k = (q & 7) * 8;
    h8 first, second, tfirst, tsecond;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const float v = tile[line][k + u], w = tile[k + u][line];
      first[u] = (half)v;
      second[u] = (half)(v - (float)first[u]);
      tfirst[u] = (half)w;
      tsecond[u] = (half)(w - (float)tfirst[u]);
    }
    const long long at = pair_at(i0 + line, t.np, j0 + k), tat = pair_at(j0 + line, t.mp, i0 + k);
    *reinterpret_cast<h8*>(r.x + at) = first;
    *reinterpret_cast<h8*>(r.x + at + 32) = second;
    *reinterpret_cast<h8*>(r.xt + tat) = tfirst;
    *reinterpret_cast<h8*>(r.xt + tat + 32) = tsecond;
  }
}

// ------------------------------------------------------------------------------------------ products

struct TileOf {
  unsigned matrix, split, tile;
  int row, col;                        // its first row and column
  bool mirror;                         // of a symmetric product, off the diagonal
};
template <int T, int PHASE>
__device__ __forceinline__ unsigned tiles_of(const DenseEntry& t) {
  const unsigned tm = t.mp / T;
  return PHASE < 2 ? tm * (tm + 1) / 2 : tm * (t.np / T);
}
template <int T, int PHASE>
__device__ __forceinline__ TileOf tile_of(const DenseEntry& t, unsigned local, unsigned splits) {
  const unsigned tiles = tiles_of<T, PHASE>(t), tm = t.mp / T;
  TileOf o;
  o.matrix = local / (tiles * splits);
  o.split = local / tiles % splits;
  o.tile = local % tiles;
  unsigned i = 0, j = o.tile;
  if constexpr (PHASE < 2) {
    while (j >= tm - i) {
      j -= tm - i;
      ++i;
    }
    j += i;
  } else {
    i = o.tile % tm;
    j = o.tile / tm;
  }
  o.row = (int)i * T;
  o.col = (int)j * T;
  o.mirror = PHASE < 2 && i != j;
  return o;
}

// Sixteen consecutive values of a row as pairs: half of a piece of 32
__device__ __forceinline__ void put_pairs(half* at, const float (&v)[16]) {
#pragma unroll
  for (int k = 0; k < 16; k += 8) {
    h8 first, second;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      first[u] = (half)v[k + u];
      second[u] = (half)(v[k + u] - (float)first[u]);
    }
    *reinterpret_cast<h8*>(at + k) = first;
    *reinterpret_cast<h8*>(at + k + 32) = second;
  }
}
__device__ __forceinline__ void get_pairs(const half* at, float (&v)[16]) {
#pragma unroll
  for (int k = 0; k < 16; k += 8) {
    const h8 first = *reinterpret_cast<const h8*>(at + k), second = *reinterpret_cast<const h8*>(at + k + 32);
#pragma unroll
    for (int u = 0; u < 8; ++u) v[k + u] = (float)first[u] + (float)second[u];
  }
}
// A matrix's step for 16 consecutive values, `count` of which are there
__device__ __forceinline__ void step_values(const DenseEntry& t, float* p, int count, const float (&x)[16]) {
  typedef v4f loose __attribute__((aligned(4)));
  const float move = t.move * (1.f / kX);
  if (count >= 16) {
    v4f q[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) q[k] = *reinterpret_cast<const loose*>(p + 4 * k);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
      for (int u = 0; u < 4; ++u) q[k][u] = fmaf(q[k][u], t.keep, -move * x[4 * k + u]);
      *reinterpret_cast<loose*>(p + 4 * k) = q[k];
    }
  } else {
#pragma unroll
    for (int k = 0; k < 16; ++k)
      if (k < count) p[k] = fmaf(p[k], t.keep, -move * x[k]);
  }
}
__device__ __forceinline__ void wave_fence() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// What becomes of a 32 x 32 piece of a sum.  Its values go through a wave's own LDS, so that memory is read and written in
// 16-byte pieces along rows, and along columns for the array by columns (for A and B the mirror).
constexpr int kTurn = 32 * 33;         // floats of it
template <int PHASE>
__device__ __forceinline__ void finish(const DenseEntry& t, const Region& r, const TileOf& o, const MuonScalars& c, int it, int row0,
                                       int col0, const v16f& acc, float* turn) {
  const int lane = threadIdx.x & 63, line = lane >> 1, part = (lane & 1) * 16;
  wave_fence();
#pragma unroll
  for (int q = 0; q < 16; ++q) turn[(8 * (q / 4) + 4 * (lane >> 5) + q % 4) * 33 + (lane & 31)] = acc[q];
  wave_fence();
  float v[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = turn[line * 33 + part + k];
  const bool over = PHASE == 2 && it + 1 >= c.iterations, tall = t.rows > t.cols;
  if constexpr (PHASE == 0) {
    half* const at = r.a + pair_at(row0 + line, t.mp, col0 + part);
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] *= kA / (kX * kX);
    put_pairs(at, v);
  } else if constexpr (PHASE == 1) {
    float a[16];
    get_pairs(r.a + pair_at(row0 + line, t.mp, col0 + part), a);
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = fmaf(c.b * (kB / kA), a[k], c.c * (kB / (kA * kA)) * v[k]);
    put_pairs(r.b + pair_at(row0 + line, t.mp, col0 + part), v);
  } else {
    half* const at = r.x + pair_at(row0 + line, t.np, col0 + part);
    float x[16];
    get_pairs(at, x);
#pragma unroll
    for (int k = 0; k < 16; ++k) v[k] = fmaf(c.a, x[k], v[k] * (1.f / kB));
    if (!over) {
      put_pairs(at, v);
    } else if (!tall) {
      if (row0 + line < t.m)
        step_values(t, t.p + ((long long)o.matrix * t.rows + row0 + line) * t.cols + col0 + part, t.n - col0 - part, v);
      return;
    }
  }
  if (PHASE < 2 && !o.mirror) return;
  wave_fence();
#pragma unroll
  for (int k = 0; k < 16; ++k) turn[line * 33 + part + k] = v[k];
  wave_fence();
#pragma unroll
  for (int k = 0; k < 16; ++k) v[k] = turn[(part + k) * 33 + line];
  if constexpr (PHASE == 2) {
    if (!over) put_pairs(r.xt + ((it + 1) & 1) * r.next + pair_at(col0 + line, t.mp, row0 + part), v);
    else if (col0 + line < t.n)
      step_values(t, t.p + ((long long)o.matrix * t.rows + col0 + line) * t.cols + row0 + part, t.m - row0 - part, v);
  } else {
    put_pairs((PHASE == 0 ? r.a : r.b) + pair_at(col0 + line, t.mp, row0 + part), v);
  }
}

template <int T>
__device__ __forceinline__ long long partial_at(unsigned local) { return (long long)local * T * T; }


// Waits until a wave has read all it asked for from LDS and at most COUNT of its loads are on their way.  (The fence of a barrier
// waits for all loads.)
template <int COUNT>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(COUNT) : "memory");
}
// (the same matrices, all in tiles of 128: 1430 us with three stages, 1469 with four, 1311 with two, which leave room for two blocks a
// compute unit)
template <int T> constexpr int kStages = T == 64 ? 4 : 2;

// A T x T tile, or a share of its sum.  PHASE 0: A = X X^T; 1: B = b A + c A A; 2: X = a X + B X.
template <int T, int PHASE>
__global__ __launch_bounds__(kThreads) void dense_product_kernel(DenseList l, MuonScalars c, int it, unsigned blocks) {
  constexpr int W = T / 2, N = W / 32, LINE = 128, SIDE = T * LINE;       // a wave's share of the tile; bytes of an operand in LDS
  constexpr int STAGES = kStages<T>, LOADS = T / 16;                      // steps in LDS or on their way; a wave's loads of one
  __shared__ __align__(16) char lds[STAGES][2 * SIDE];
  float scale;
  if (!muon_scale(c, scale)) return;
  // an XCD has a contiguous share of the tiles, whose operands overlap: they stay in its L2
  const unsigned item = (unsigned)xcd_contiguous_item(blockIdx.x, gridDim.x);
  if (item >= blocks) return;
  int e = 0;
  while (e + 1 < l.count && l.t[e + 1].first[PHASE] <= item) ++e;
  const DenseEntry& t = l.t[e];
  const unsigned local = item - t.first[PHASE], splits = t.splits[PHASE];
  const TileOf o = tile_of<T, PHASE>(t, local, splits);
  const Region r = region_of(t, o.matrix);
  const int inner = PHASE == 0 ? t.np : t.mp, steps = inner / kStep, share = (steps + (int)splits - 1) / (int)splits;
  const int s0 = (int)o.split * share, s1 = s0 + share < steps ? s0 + share : steps;
  const half* const left = PHASE == 0 ? r.x : PHASE == 1 ? r.a : r.b;
  const half* const right = PHASE == 0 ? r.x : PHASE == 1 ? r.a : r.xt + (it & 1) * r.next;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // to LDS: a wave's instruction takes eight rows; piece p of row i goes to place p ^ (i / 2 % 8)
  const int piece = (lane & 7) ^ ((lane >> 4) | ((w & 1) << 2));
  const long long lane_at = (long long)(w * 8 + (lane >> 3)) * 2 * inner + piece * 8;
  const half* lp = left + (long long)o.row * 2 * inner + lane_at + (long long)s0 * 64;
  const half* rp = right + (long long)o.col * 2 * inner + lane_at + (long long)s0 * 64;
  auto load = [&](int buffer) {
#pragma unroll
    for (int u = 0; u < T / 32; ++u) {
      const long long down = (long long)u * 32 * 2 * inner;
      char* const to = lds[buffer] + (u * 4 + w) * 1024;
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(lp + down),
                                       (__attribute__((address_space(3))) void*)to, 16, 0, 0);
      __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(rp + down),
                                       (__attribute__((address_space(3))) void*)(to + SIDE), 16, 0, 0);
    }
    lp += 64;
    rp += 64;
  };
  const int wr = (w >> 1) * W, wc = (w & 1) * W;
  int at[2][2];                        // [half of the step][part]
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int q = 0; q < 2; ++q) at[h][q] = (lane & 31) * LINE + (((q * 4 + h * 2 + (lane >> 5)) ^ ((lane >> 1) & 7)) << 4);

  v16f acc[N][N];
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[i][j][q] = 0.f;
  for (int k = 0; k < STAGES - 1; ++k)
    if (s0 + k < s1) load(k);
  for (int s = s0; s < s1; ++s) {
    const int buffer = (s - s0) % STAGES, ahead = s1 - 1 - s;              // steps after this one: STAGES - 2 of them are on their way
    if (STAGES > 3 && ahead >= 2) wait_loads<2 * LOADS>();
    else if (STAGES > 2 && ahead >= 1) wait_loads<LOADS>();
    else wait_loads<0>();
    // this wave's pieces of the step are there; with the barrier all waves' are, and all waves are done with the step before,
    // whose buffer is the next to be filled
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (s + STAGES - 1 < s1) load((s - s0 + STAGES - 1) % STAGES);
    const char *const a = lds[buffer] + wr * LINE, *const b = lds[buffer] + SIDE + wc * LINE;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      h8 af[2][N], bf[2][N];
#pragma unroll
      for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          af[q][i] = *reinterpret_cast<const h8*>(a + at[h][q] + i * 32 * LINE);
          bf[q][i] = *reinterpret_cast<const h8*>(b + at[h][q] + i * 32 * LINE);
        }
#pragma unroll
      for (int q = 0; q < 3; ++q)
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
          for (int j = 0; j < N; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(af[q == 2][i], bf[q == 1][j], acc[i][j], 0, 0, 0);
    }
  }
  if (splits > 1) {                    // in the order of the registers, which the launch that adds them shares
    float* const to = l.part + t.part_at[PHASE] + partial_at<T>(local) + w * (T * T / 4) + lane * 4;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
      for (int j = 0; j < N; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q)
          *reinterpret_cast<v4f*>(to + ((i * N + j) * 4 + q) * 256) =
              v4f{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    return;
  }
  __syncthreads();
  float* const turn = reinterpret_cast<float*>(lds[0]) + w * kTurn;
  static_assert(4 * kTurn * sizeof(float) <= sizeof(lds), "the operands' LDS is used again");
#pragma unroll
  for (int i = 0; i < N; ++i)
#pragma unroll
    for (int j = 0; j < N; ++j) finish<PHASE>(t, r, o, c, it, o.row + wr + i * 32, o.col + wc + j * 32, acc[i][j], turn);
}

// Adds the shares of the tiles whose sums are split, in their order; a block takes one 32 x 32 piece of every wave's.
template <int T, int PHASE>
__global__ __launch_bounds__(kThreads) void dense_sum_kernel(DenseList l, MuonScalars c, int it) {
  constexpr int W = T / 2, N = W / 32;
  __shared__ float turns[4][kTurn];
  float scale;
  if (!muon_scale(c, scale)) return;
  const unsigned block = blockIdx.x / (N * N), i = blockIdx.x / N % N, j = blockIdx.x % N;
  int k = 0;
  while (k + 1 < l.count && l.t[k + 1].first_sum[PHASE] <= block) ++k;
  const DenseEntry& t = l.t[k];
  const unsigned local = block - t.first_sum[PHASE], tiles = tiles_of<T, PHASE>(t), splits = t.splits[PHASE];
  const TileOf o = tile_of<T, PHASE>(t, local, 1);
  const Region r = region_of(t, o.matrix);
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wr = (w >> 1) * W, wc = (w & 1) * W;
  const float* const from = l.part + t.part_at[PHASE] + partial_at<T>(o.matrix * splits * tiles + o.tile) + w * (T * T / 4) + lane * 4 +
                            (i * N + j) * 1024;
  v4f v[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) v[q] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (unsigned n = 0; n < splits; ++n) {
    const float* const at = from + partial_at<T>(n * tiles);
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] += *reinterpret_cast<const v4f*>(at + q * 256);
  }
  v16f acc;
#pragma unroll
  for (int q = 0; q < 16; ++q) acc[q] = v[q / 4][q % 4];
  finish<PHASE>(t, r, o, c, it, o.row + wr + (int)i * 32, o.col + wc + (int)j * 32, acc, turns[w]);
}

// ------------------------------------------------------------------------------------------ launches

constexpr long long kGroupBytes = 1ll << 30;     // scratch of the matrices that go through their launches together, where they are several
constexpr unsigned kMostBlocks = 1u << 22;       // of a launch
// 4 x 1024 x 1024, 1024 x 4096, 4096 x 1024 and 1000 x 1536 together: 1277 us with 256 blocks wanted, 1311 with 512, 1470 with 1024;
// shares of 16 or 32 steps at least are slower too.
constexpr int kWantBlocks = 256, kLeastSteps = 8;

long long tiles_host(long long mp, long long np, int T, int phase) {
  const long long tm = mp / T;
  return phase < 2 ? tm * (tm + 1) / 2 : tm * (np / T);
}
int padded(int v, int T) { return (v + T - 1) / T * T; }

// The next matrices of the list, from matrix `done` of tensor k on, that go together: entries with all but their addresses in
// scratch, whose bytes are returned.
struct Group {
  DenseList l;
  long long bytes;
  unsigned pieces, tiles, blocks[3], sums[3];
};
bool is_dense(const MuonTensor& t) { return !t.modes && !muon_is_small(t); }

// Tiles of 128 read half as much for a product, and are worth it for matrices that have a few of them on a side, where all tensors together
// fill the chip with them.  us a step with tiles of 64 and of 128: 1024 x 4096 481 and 420, eight of 1024 x 1024 912 and 788, 32 of
// 512 x 512 562 and 529, but four of 1024 x 1024 526 and 541, 16 of 512 x 512 336 and 400, 64 of 192 x 192 172 and 244.
constexpr int kNarrowSide = 192;
int shorter_side(const MuonTensor& t) { return t.rows < t.cols ? t.rows : t.cols; }
bool tiles_of_128(const MuonTensor* t, int count) {
  double steps = 0.0;
  for (int k = 0; k < count; ++k) {
    const int m = shorter_side(t[k]), n = t[k].rows + t[k].cols - m;
    if (is_dense(t[k]) && m > kNarrowSide) steps += (double)t[k].batch * (double)tiles_host(padded(m, 128), 0, 128, 0) * (padded(n, 128) / kStep);
  }
  return steps >= 4500.0;
}

template <int T>
bool next_group(const MuonTensor* t, int count, bool wide, double lr, int& k, long long& done, Group* g) {
  g->l.count = 0;
  g->bytes = 0;
  long long part = 0;
  for (; k < count && g->l.count < kPerLaunch; ++k, done = 0) {
    if (!is_dense(t[k]) || (wide && shorter_side(t[k]) > kNarrowSide) != (T == 128)) continue;
    const bool tall = t[k].rows > t[k].cols;
    DenseEntry e{};
    e.rows = t[k].rows;
    e.cols = t[k].cols;
    e.m = tall ? t[k].cols : t[k].rows;
    e.n = tall ? t[k].rows : t[k].cols;
    e.mp = padded(e.m, T);
    e.np = padded(e.n, T);
    e.region = (region_bytes(e.mp, e.np) + 255) / 256 * 256;
    long long fit = (kGroupBytes - g->bytes) / e.region;
    const long long tiles = tiles_host(e.mp, e.np, 64, 2), room = kMostBlocks / (2 * tiles * kPerLaunch);
    if (fit > room) fit = room;
    if (fit < 1) {
      if (g->l.count > 0) break;
      fit = 1;
    }
    const long long here = t[k].batch - done < fit ? t[k].batch - done : fit;
    const long long values = (long long)e.rows * e.cols, first = done * values;
    e.p = t[k].p + first;
    e.g = t[k].g + first;
    e.mom = t[k].m + first;
    e.ws = reinterpret_cast<char*>(g->bytes);
    e.run = ((values + kPieces - 1) / kPieces + kPieceValues - 1) / kPieceValues * kPieceValues;
    e.pieces = (unsigned)((values + e.run - 1) / e.run);
    e.count = (unsigned)here;
    e.keep = (float)(1.0 - lr * t[k].decay);
    e.move = (float)(lr * t[k].scale);
    g->bytes += here * e.region;
    g->l.t[g->l.count++] = e;
    done += here;
    if (done < t[k].batch) break;
  }
  if (g->l.count == 0) return false;
  g->pieces = g->tiles = 0;
  for (int i = 0; i < g->l.count; ++i) {
    DenseEntry& e = g->l.t[i];
    e.first_piece = g->pieces;
    e.first_tile = g->tiles;
    g->pieces += e.count * e.pieces;
    g->tiles += e.count * (unsigned)(e.mp / 64) * (unsigned)(e.np / 64);
  }
  for (int phase = 0; phase < 3; ++phase) {
    // sums are split so that all tiles together make about kWantBlocks blocks of as many steps each
    double work = 0.0;
    for (int i = 0; i < g->l.count; ++i) {
      const DenseEntry& e = g->l.t[i];
      work += (double)e.count * tiles_host(e.mp, e.np, T, phase) * ((phase == 0 ? e.np : e.mp) / kStep);
    }
    double each = work / kWantBlocks;
    if (each < kLeastSteps) each = kLeastSteps;
    g->blocks[phase] = g->sums[phase] = 0;
    long long floats = 0;
    for (int i = 0; i < g->l.count; ++i) {
      DenseEntry& e = g->l.t[i];
      const long long tiles = tiles_host(e.mp, e.np, T, phase) * e.count, steps = (phase == 0 ? e.np : e.mp) / kStep;
      long long splits = (long long)((double)steps / each + 0.5);
      splits = splits < 1 ? 1 : splits > 64 ? 64 : splits;
      splits = (steps + (steps + splits - 1) / splits - 1) / ((steps + splits - 1) / splits);       // none of them empty
      e.splits[phase] = (unsigned)splits;
      e.first[phase] = g->blocks[phase];
      e.first_sum[phase] = g->sums[phase];
      g->blocks[phase] += (unsigned)(tiles * splits);
      e.part_at[phase] = floats;
      if (splits > 1) {
        g->sums[phase] += (unsigned)tiles;
        floats += tiles * splits * T * T;
      }
    }
    part = floats > part ? floats : part;
  }
  g->l.part = reinterpret_cast<float*>(g->bytes);
  g->bytes += part * (long long)sizeof(float);
  return true;
}

template <int T, int PHASE>
hipError_t launch_product(const Group& g, const MuonScalars& c, int it, hipStream_t s) {
  hipLaunchKernelGGL((dense_product_kernel<T, PHASE>), dim3((g.blocks[PHASE] + 7) / 8 * 8), dim3(kThreads), 0, s, g.l, c, it, g.blocks[PHASE]);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || g.sums[PHASE] == 0) return e;
  hipLaunchKernelGGL((dense_sum_kernel<T, PHASE>), dim3(g.sums[PHASE] * (T / 64) * (T / 64)), dim3(kThreads), 0, s, g.l, c, it);
  return hipGetLastError();
}
template <int T>
hipError_t launch_group(Group& g, const MuonScalars& c, void* ws, hipStream_t s) {
  for (int i = 0; i < g.l.count; ++i) g.l.t[i].ws = static_cast<char*>(ws) + reinterpret_cast<uintptr_t>(g.l.t[i].ws);
  g.l.part = reinterpret_cast<float*>(static_cast<char*>(ws) + reinterpret_cast<uintptr_t>(g.l.part));
  hipLaunchKernelGGL(dense_momentum_kernel, dim3(g.pieces), dim3(kThreads), 0, s, g.l, c);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(dense_parts_kernel, dim3(g.tiles), dim3(kThreads), 0, s, g.l, c);
  e = hipGetLastError();
  for (int it = 0; it < c.iterations && e == hipSuccess; ++it) {
    e = launch_product<T, 0>(g, c, it, s);
    if (e == hipSuccess) e = launch_product<T, 1>(g, c, it, s);
    if (e == hipSuccess) e = launch_product<T, 2>(g, c, it, s);
  }
  return e;
}
template <int T>
hipError_t launch_side(const MuonTensor* t, int count, const MuonScalars& c, double lr, void* ws, hipStream_t s) {
  const bool wide = tiles_of_128(t, count);
  int k = 0;
  long long done = 0;
  for (Group g; next_group<T>(t, count, wide, lr, k, done, &g);) {
    const hipError_t e = launch_group<T>(g, c, ws, s);
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}
template <int T>
size_t side_bytes(const MuonTensor* t, int count) {
  const bool wide = tiles_of_128(t, count);
  size_t most = 0;
  int k = 0;
  long long done = 0;
  for (Group g; next_group<T>(t, count, wide, 0.0, k, done, &g);) most = (size_t)g.bytes > most ? (size_t)g.bytes : most;
  return most;
}

}  // namespace

size_t muon_dense_bytes(const MuonTensor* t, int count) {
  const size_t a = side_bytes<128>(t, count), b = side_bytes<64>(t, count);
  return a > b ? a : b;
}

hipError_t launch_muon_dense(const MuonTensor* t, int count, const MuonScalars& c, double lr, void* ws, hipStream_t s) {
  const hipError_t e = launch_side<128>(t, count, c, lr, ws, s);
  return e != hipSuccess ? e : launch_side<64>(t, count, c, lr, ws, s);
}

}  // namespace fno
