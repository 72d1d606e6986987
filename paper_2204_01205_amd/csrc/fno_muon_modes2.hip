// The Muon step of spectral weights with 5 to 8 channels on either side: two tiles of 4 x 4 by two, four modes a wave.
//
// The weights of such a network are small (8 channels, 1536 modes: 0.8 MB), and what counts is the time that five iterations of three
// dependent products take: 0.9 us each (fno_muon_modes.hip, with six barriers: 2.0).  The 16 outer products of a v_mfma_f32_4x4x1 are
// four modes times their four tiles, so that a product of eight steps is 32 instructions, and nothing waits for another wave.  Lane 16
// s + 4 md + j: tile (s / 2, s % 2), mode md, column (or row) j of the tile; a register is a row.  X, A = X X^H and B = a + b A + c A A
// have a place each in a wave's LDS, [row][column][mode] with four places of padding a row: rows and columns of a tile are read without
// bank conflicts.
#include "fno_muon_modes.h"

namespace fno {

namespace {

constexpr int kRows = 8, kPitch = 4 * kRows + 4, kMatrix = kRows * kPitch;        // places
constexpr int kWaveModes = 4, kWaves = 4;
constexpr int kPerLaunch = 32;

struct Modes2Entry {
  float2* p;
  const float2* g;
  float2* mom;
  long long modes;
  unsigned first;                      // first block of the launch that belongs to this tensor
  int m, n;
  float keep, move;                    // 1 - lr weight_decay, lr scale
};
struct Modes2List {
  Modes2Entry t[kPerLaunch];
  int count;
  unsigned blocks;
};

// LDS accesses of a wave are worked in order; this keeps the compiler to it.
__device__ __forceinline__ void in_order() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

__global__ __launch_bounds__(64 * kWaves) void muon_modes2_kernel(Modes2List l, MuonScalars c) {
  __shared__ float2 lds[kWaves][3 * kMatrix];
  const unsigned item = (unsigned)xcd_contiguous_item(blockIdx.x, gridDim.x);
  if (item >= l.blocks) return;
  float scale;
  if (!muon_scale(c, scale)) return;
  int k = 0;
  while (k + 1 < l.count && l.t[k + 1].first <= item) ++k;
  const Modes2Entry& t = l.t[k];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 3, md = (lane >> 2) & 3;
  const int I = lane >> 5, J = (lane >> 4) & 1, row0 = 4 * I, col = 4 * J + j;
  float2 *const X = lds[w], *const A = X + kMatrix, *const B = A + kMatrix;
  const long long mode = ((long long)(item - t.first) * kWaves + w) * kWaveModes + md;
  const bool here = mode < t.modes && col < t.n;

  // What lies past the matrix or the last mode is read from its last place, becomes a zero that stays one, and is not stored.
  long long at[4];
  bool in[4];
  float2 x[4];
  {
    float2 o[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int i = row0 + r < t.m ? row0 + r : t.m - 1, q = col < t.n ? col : t.n - 1;
      at[r] = ((long long)i * t.n + q) * t.modes + (mode < t.modes ? mode : t.modes - 1);
      in[r] = here && row0 + r < t.m;
      x[r] = t.g[at[r]];
      o[r] = t.mom[at[r]];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float2 u = make_float2(muon_momentum(c, x[r].x * scale, o[r].x), muon_momentum(c, x[r].y * scale, o[r].y));
      x[r] = in[r] ? u : make_float2(0.f, 0.f);
      if (in[r]) t.mom[at[r]] = o[r];
    }
  }
  {
    double sum = 0.0;
#pragma unroll
    for (int r = 0; r < 4; ++r) sum = fma((double)x[r].x, (double)x[r].x, fma((double)x[r].y, (double)x[r].y, sum));
    sum += __shfl_xor(sum, 1);
    sum += __shfl_xor(sum, 2);
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    const double inv = muon_inverse(sum, c.eps);
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = make_float2((float)(x[r].x * inv), (float)(x[r].y * inv));
  }

  const int own = row0 * kPitch + 4 * col + md;                        // element (4 I + r, 4 J + j): r rows on
  auto by_row = [&](int tile) { return (4 * tile + j) * kPitch + md; };          // element (4 tile + j, 0)
  auto by_col = [&](int tile) { return (4 * tile + j) * 4 + md; };               // element (0, 4 tile + j)
  for (int it = 0; it < c.iterations; ++it) {
    in_order();
#pragma unroll
    for (int r = 0; r < 4; ++r) X[own + r * kPitch] = x[r];
    in_order();
    // A(I, J) = sum over columns n of X(I, n) conj X(J, n)
    Tile4 q;
    clear(q);
    {
      float2 a[kRows], b[kRows];
#pragma unroll
      for (int n = 0; n < kRows; ++n) {
        a[n] = X[by_row(I) + 4 * n];
        b[n] = X[by_row(J) + 4 * n];
      }
#pragma unroll
      for (int n = 0; n < kRows; ++n) add_conj_right(q, a[n], b[n]);
    }
    q.i -= q.h;
    in_order();
#pragma unroll
    for (int r = 0; r < 4; ++r) A[own + r * kPitch] = make_float2(q.r[r], q.i[r]);
    in_order();
    // B = a + b A + c A A, (A A)(I, J) = sum over rows n of conj A(n, I) A(n, J)
    Tile4 u;
    clear(u);
    {
      float2 a[kRows], b[kRows];
#pragma unroll
      for (int n = 0; n < kRows; ++n) {
        a[n] = A[by_col(I) + n * kPitch];
        b[n] = A[by_col(J) + n * kPitch];
      }
#pragma unroll
      for (int n = 0; n < kRows; ++n) add_conj_left(u, a[n], b[n]);
    }
    in_order();
#pragma unroll
    for (int r = 0; r < 4; ++r)
      B[own + r * kPitch] = make_float2(fmaf(c.b, q.r[r], c.c * u.r[r]) + (I == J && r == j ? c.a : 0.f),
                                        fmaf(c.b, q.i[r], c.c * (u.i[r] - u.h[r])));
    in_order();
    // X(I, J) = sum over rows n of conj B(n, I) X(n, J)
    clear(u);
    {
      float2 a[kRows], b[kRows];
#pragma unroll
      for (int n = 0; n < kRows; ++n) {
        a[n] = B[by_col(I) + n * kPitch];
        b[n] = X[by_col(J) + n * kPitch];
      }
#pragma unroll
      for (int n = 0; n < kRows; ++n) add_conj_left(u, a[n], b[n]);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] = make_float2(u.r[r], u.i[r] - u.h[r]);
  }

  float2 p[4];
#pragma unroll
  for (int r = 0; r < 4; ++r) p[r] = t.p[at[r]];
#pragma unroll
  for (int r = 0; r < 4; ++r)
    if (in[r]) t.p[at[r]] = make_float2(fmaf(p[r].x, t.keep, -t.move * x[r].x), fmaf(p[r].y, t.keep, -t.move * x[r].y));
}

}  // namespace

// us a step of 8 x 8, here and in fno_muon_modes.hip: 1536 modes 11 and 16, 24576 32 and 39, 49152 51 and 55, 110592 125 and 109 (there half
// of a Hermitian product's tiles are mirrored, here all four are worked out, and all a wave has are four modes of a cache line).
bool muon_is_modes2(const MuonTensor& t) {
  return t.modes && t.rows > 4 && t.rows <= 8 && t.cols > 4 && t.cols <= 8 && t.batch <= 65536;
}

// 32 tensors a launch: 2^17 blocks at most.
hipError_t launch_muon_modes2(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s) {
  constexpr int kModes = kWaves * kWaveModes;
  Modes2List l;
  l.count = 0;
  l.blocks = 0;
  auto flush = [&]() {
    if (l.count > 0) hipLaunchKernelGGL(muon_modes2_kernel, dim3((l.blocks + 7) / 8 * 8), dim3(64 * kWaves), 0, s, l, c);
    const hipError_t e = l.count > 0 ? hipGetLastError() : hipSuccess;
    l.count = 0;
    l.blocks = 0;
    return e;
  };
  for (int k = 0; k < count; ++k) {
    if (!muon_is_modes2(t[k])) continue;
    if (l.count == kPerLaunch) {
      const hipError_t e = flush();
      if (e != hipSuccess) return e;
    }
    l.t[l.count++] = Modes2Entry{reinterpret_cast<float2*>(t[k].p), reinterpret_cast<const float2*>(t[k].g),
                                 reinterpret_cast<float2*>(t[k].m), (long long)t[k].batch, l.blocks, t[k].rows, t[k].cols,
                                 (float)(1.0 - lr * t[k].decay), (float)(lr * t[k].scale)};
    l.blocks += (unsigned)((t[k].batch + kModes - 1) / kModes);
  }
  return flush();
}

}  // namespace fno
