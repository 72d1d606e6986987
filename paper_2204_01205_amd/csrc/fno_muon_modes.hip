// The Muon step of spectral weights: one complex matrix X, m x n with m <= n <= 32, for every kept mode.
//
// A block takes 16 modes through the whole step: momentum, normalisation, all iterations, weights; memory sees every tensor
// once.  Products run on v_mfma_f32_4x4x1, whose 16 independent 4 x 4 outer products are 16 modes: widths need whole fours
// only (20 is five; tiles of 16 or 32 would be two or three times the work), and neighbouring modes lie side by side in memory.  A
// lane is (mode, column of a tile), a register a row.  Wave J of a block owns the columns of tile J of X, in registers.  An
// iteration, with A and B Hermitian, so that a row of either is the conjugate of a column:
//   A = X X^H and B = a + b A + c A A: wave J takes the tiles (J, J .. J + m/8), around the corner, of which the other half are
//   the mirrors, operands from LDS (X by rows, A by columns);
//   X = B X: its own columns, B from LDS.
// Matrix instructions bound it: 110592 modes of 16 x 16 take 86 us an iteration, of which these are 52; the rest are the waits of a block's
// waves for each other and for LDS.  Loads and stores alone take 275 us (4.1 TB/s).  Beyond 20 channels a compute unit has room for two
// blocks or, from 25 on, for one (101 to 131 KB), which all wait at a barrier: 24 channels take 329 us an iteration, 32 channels 593.  (With 25 to 32
// on the shorter side two of 256 registers are spilled, 12 bytes a lane.)
// X, A and B take turns in one LDS buffer, [row][tile][mode][column] with one entry of padding a row: a tile read by columns
// is contiguous, one read by rows has its four rows in neighbouring banks.
#include "fno_muon_modes.h"

namespace fno {

namespace {

constexpr int kModes = 16;             // modes of a block
constexpr int kPerLaunch = 32;         // tensors whose addresses go with one launch's arguments

struct ModesEntry {
  float2* p;
  const float2* g;
  float2* mom;
  long long modes, si, sj;             // si, sj: distance of rows and columns of X, in values
  unsigned first, skip;                // first block of the launch that belongs to this tensor; blocks of it in earlier launches
  int m, n;
  float keep, move;                    // 1 - lr weight_decay, lr scale
};
struct ModesList {
  ModesEntry t[kPerLaunch];
  int count;
  unsigned blocks;
};

// A place that the compiler takes for a new one: it would keep the addresses of all rows between the loads and the stores.
__device__ __forceinline__ long long opaque_place(long long at) {
  asm volatile("" : "+v"(at));
  return at;
}

template <int TM>
__global__ __launch_bounds__(512) void muon_modes_kernel(ModesList l, MuonScalars c) {
  constexpr int M = 4 * TM, ND = TM / 2 + 1, RA = 64 * TM + 1;
  extern __shared__ float2 lds[];
  const unsigned item = (unsigned)xcd_contiguous_item(blockIdx.x, gridDim.x);
  if (item >= l.blocks) return;
  float scale;
  if (!muon_scale(c, scale)) return;
  int k = 0;
  while (k + 1 < l.count && l.t[k + 1].first <= item) ++k;
  const ModesEntry& t = l.t[k];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), TN = blockDim.x >> 6;
  const int RX = 64 * TN + 1;
  const int b = lane >> 2, j = lane & 3, col = 4 * w + j;
  const long long mode = ((long long)(item - t.first) + t.skip) * kModes + b;
  const bool here = mode < t.modes && col < t.n;
  const long long at = (col < t.n ? col : t.n - 1) * t.sj + (mode < t.modes ? mode : t.modes - 1);

  // What lies past the matrix or the last mode is a zero that stays one and is not stored; of rows, the last three may.
  float xr[M], xi[M];
  {
    constexpr int PART = TM > 4 ? M / 2 : M;               // rows that are on their way at a time: registers
    const float2 *gp = t.g + at, *mp = t.mom + at;
    float2* to = t.mom + at;
#pragma unroll
    for (int part = 0; part < M; part += PART) {
      float2 g[PART], o[PART];
#pragma unroll
      for (int i = 0; i < PART; ++i) {
        g[i] = *gp;
        o[i] = *mp;
        if (part + i < M - 4 || part + i + 1 < t.m) {
          gp += t.si;
          mp += t.si;
        }
      }
#pragma unroll
      for (int i = 0; i < PART; ++i) {
        const float ur = muon_momentum(c, g[i].x * scale, o[i].x), ui = muon_momentum(c, g[i].y * scale, o[i].y);
        const bool in = here && (part + i < M - 3 || part + i < t.m);
        xr[part + i] = in ? ur : 0.f;
        xi[part + i] = in ? ui : 0.f;
      }
      if (here) {
        to = t.mom + opaque_place(to - t.mom);
#pragma unroll
        for (int i = 0; i < PART; ++i) {
          if (part + i < M - 3 || part + i < t.m) *to = o[i];
          to += t.si;
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  {
    // |u|^2 in float where that holds its squares, else in double
    auto total = [&](auto zero) {
      typedef decltype(zero) real;
      real sum = zero;
#pragma unroll
      for (int i = 0; i < M; ++i) {
        sum += (real)xr[i] * (real)xr[i];
        sum += (real)xi[i] * (real)xi[i];
      }
      sum += __shfl_xor(sum, 1);
      sum += __shfl_xor(sum, 2);
      real* const red = reinterpret_cast<real*>(lds);
      __syncthreads();
      if (j == 0) red[w * kModes + b] = sum;
      __syncthreads();
      sum = zero;
      for (int v = 0; v < TN; ++v) sum += red[v * kModes + b];
      return sum;
    };
    auto times = [&](auto by) {
#pragma unroll
      for (int i = 0; i < M; ++i) {
        xr[i] = (float)(xr[i] * by);
        xi[i] = (float)(xi[i] * by);
      }
    };
    const float squares = total(0.f);
    // (a matrix takes its own way, whatever its neighbours are)
    const bool plain = squares > 1e-28f && squares < 1e30f;
    const float inv = 1.0f / (sqrtf(squares) + (float)c.eps);
    if (__all(plain)) {
      times(inv);
    } else {
      const double fine = muon_inverse(total(0.0), c.eps);
      times(plain ? (double)inv : fine);
    }
  }

  for (int it = 0; it < c.iterations; ++it) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < M; ++i) lds[i * RX + w * 64 + lane] = make_float2(xr[i], xi[i]);
    __syncthreads();
    v4f ar[ND], ai[ND];
    int tile[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      ar[d] = ai[d] = v4f{0.f, 0.f, 0.f, 0.f};
      tile[d] = w + d < TM ? w + d : w + d - TM;
    }
    // A(w, J) = sum over columns k of X(w, k) conj X(J, k)
    if (w < TM) {
      const float2* row[ND];
#pragma unroll
      for (int d = 0; d < ND; ++d) row[d] = lds + (4 * tile[d] + j) * RX + 4 * b;
      for (int kt = 0; kt < TN; ++kt) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float2 v[ND];
#pragma unroll
          for (int d = 0; d < ND; ++d) v[d] = row[d][kt * 64 + q];
          const float nr = -v[0].x;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            ar[d] = mfma4(v[0].x, v[d].x, ar[d]);
            ai[d] = mfma4(v[0].y, v[d].x, ai[d]);
          }
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            ar[d] = mfma4(v[0].y, v[d].y, ar[d]);
            ai[d] = mfma4(nr, v[d].y, ai[d]);
          }
        }
      }
    }
    // a tile and its mirror to LDS
    auto put = [&]() {
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        if (TM % 2 == 0 && d == TM / 2 && w >= TM / 2) continue;     // the mirror of another wave's
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          lds[(4 * w + r) * RA + tile[d] * 64 + lane] = make_float2(ar[d][r], ai[d][r]);
          if (d > 0) lds[(4 * tile[d] + j) * RA + w * 64 + 4 * b + r] = make_float2(ar[d][r], -ai[d][r]);
        }
      }
    };
    __syncthreads();
    if (w < TM) put();
    __syncthreads();
    // B = a + b A + c A A, with (A A)(w, J) = sum over k of conj A(k, w) A(k, J)
    if (w < TM) {
      const float2* colp[ND];
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        ar[d] = ai[d] = v4f{0.f, 0.f, 0.f, 0.f};
        colp[d] = lds + tile[d] * 64 + lane;
      }
      for (int kt = 0; kt < TM; ++kt) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          float2 v[ND];
#pragma unroll
          for (int d = 0; d < ND; ++d) v[d] = colp[d][(4 * kt + q) * RA];
          const float ni = -v[0].y;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            ar[d] = mfma4(v[0].x, v[d].x, ar[d]);
            ai[d] = mfma4(v[0].x, v[d].y, ai[d]);
          }
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            ar[d] = mfma4(v[0].y, v[d].y, ar[d]);
            ai[d] = mfma4(ni, v[d].x, ai[d]);
          }
        }
      }
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float2 own = colp[d][(4 * w + r) * RA];
          ar[d][r] = fmaf(c.b, own.x, c.c * ar[d][r]);
          if (d == 0) ar[d][r] += r == j ? c.a : 0.f;
          ai[d][r] = fmaf(c.b, own.y, c.c * ai[d][r]);
        }
    }
    __syncthreads();
    if (w < TM) put();
    __syncthreads();
    // X(I, w) = sum over k of conj B(k, I) X(k, w)
    v4f yr[TM], yi[TM];
#pragma unroll
    for (int I = 0; I < TM; ++I) yr[I] = yi[I] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < M; ++q) {
      float2 v[TM];
#pragma unroll
      for (int I = 0; I < TM; ++I) v[I] = lds[q * RA + I * 64 + lane];
      const float nr = -xr[q];
#pragma unroll
      for (int I = 0; I < TM; ++I) {
        yr[I] = mfma4(v[I].x, xr[q], yr[I]);
        yi[I] = mfma4(v[I].x, xi[q], yi[I]);
      }
#pragma unroll
      for (int I = 0; I < TM; ++I) {
        yr[I] = mfma4(v[I].y, xi[q], yr[I]);
        yi[I] = mfma4(v[I].y, nr, yi[I]);
      }
    }
#pragma unroll
    for (int I = 0; I < TM; ++I)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        xr[4 * I + r] = yr[I][r];
        xi[4 * I + r] = yi[I][r];
      }
  }

  if (!here) return;
  float2 p[M];
  const float2* from = t.p + at;
#pragma unroll
  for (int i = 0; i < M; ++i) {
    p[i] = *from;
    if (i < M - 4 || i + 1 < t.m) from += t.si;
  }
  float2* to = t.p + opaque_place(at);
#pragma unroll
  for (int i = 0; i < M; ++i) {
    if (i < M - 3 || i < t.m) *to = make_float2(fmaf(p[i].x, t.keep, -t.move * xr[i]), fmaf(p[i].y, t.keep, -t.move * xi[i]));
    to += t.si;
  }
}

template <int TM>
hipError_t launch_tiles(int tn, const ModesList& l, const MuonScalars& c, hipStream_t s) {
  auto rows = [](int tn) { return (size_t)4 * TM * (64 * tn + 1) * sizeof(float2); };
  const size_t bytes = rows(tn);
  const hipError_t e = ask_local_memory(reinterpret_cast<const void*>(muon_modes_kernel<TM>), bytes, rows(8));
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(muon_modes_kernel<TM>, dim3((l.blocks + 7) / 8 * 8), dim3(64 * tn), bytes, s, l, c);
  return hipGetLastError();
}
hipError_t launch_list(int tm, int tn, const ModesList& l, const MuonScalars& c, hipStream_t s) {
  switch (tm) {
    case 1: return launch_tiles<1>(tn, l, c, s);
    case 2: return launch_tiles<2>(tn, l, c, s);
    case 3: return launch_tiles<3>(tn, l, c, s);
    case 4: return launch_tiles<4>(tn, l, c, s);
    case 5: return launch_tiles<5>(tn, l, c, s);
    case 6: return launch_tiles<6>(tn, l, c, s);
    case 7: return launch_tiles<7>(tn, l, c, s);
    default: return launch_tiles<8>(tn, l, c, s);
  }
}

}  // namespace

// Tensors with as many tiles on either side go with one launch, of 2^22 blocks at most.
hipError_t launch_muon_modes(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s) {
  constexpr long long kMost = 1ll << 22;
  for (int tm = 1; tm <= 8; ++tm)
    for (int tn = tm; tn <= 8; ++tn) {
      ModesList l;
      l.count = 0;
      l.blocks = 0;
      auto flush = [&]() {
        const hipError_t e = l.count > 0 ? launch_list(tm, tn, l, c, s) : hipSuccess;
        l.count = 0;
        l.blocks = 0;
        return e;
      };
      for (int k = 0; k < count; ++k) {
        const int rows = t[k].rows, cols = t[k].cols, m = rows < cols ? rows : cols, n = rows < cols ? cols : rows;
        if (!t[k].modes || muon_is_modes5(t[k]) || muon_is_modes2(t[k]) || (m + 3) / 4 != tm || (n + 3) / 4 != tn) continue;
        const long long row = (long long)cols * t[k].batch, column = t[k].batch, blocks = (t[k].batch + kModes - 1) / kModes;
        for (long long done = 0; done < blocks;) {
          if (l.count == kPerLaunch || l.blocks == kMost) {
            const hipError_t e = flush();
            if (e != hipSuccess) return e;
          }
          const long long here = blocks - done < kMost - l.blocks ? blocks - done : kMost - l.blocks;
          l.t[l.count++] = ModesEntry{reinterpret_cast<float2*>(t[k].p), reinterpret_cast<const float2*>(t[k].g),
                                      reinterpret_cast<float2*>(t[k].m), (long long)t[k].batch, rows <= cols ? row : column,
                                      rows <= cols ? column : row, l.blocks, (unsigned)done, m, n, (float)(1.0 - lr * t[k].decay),
                                      (float)(lr * t[k].scale)};
          l.blocks += (unsigned)here;
          done += here;
        }
      }
      const hipError_t e = flush();
      if (e != hipSuccess) return e;
    }
  return hipSuccess;
}

}  // namespace fno
