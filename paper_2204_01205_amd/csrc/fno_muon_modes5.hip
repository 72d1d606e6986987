// The Muon step of spectral weights with 17 to 20 channels on either side: five tiles of 4 x 4 by five, four modes a wave.
//
// Five columns of tiles do not go evenly over the four vector units of a compute unit, and in a block that shares a mode's matrices
// every phase waits for the slowest wave (fno_muon_modes.hip takes 1563 us for five iterations of 110592 modes, of which matrix
// instructions are 540).  Here a wave has four modes to itself and nothing waits for another wave: the 16 outer products of a
// v_mfma_f32_4x4x1 are four modes times four tiles.  Lane 16 s + 4 md + j: tile slot s, mode md, column (or row) j of a tile.
//   X: columns 4 s + j of all rows in registers (`x`), and of the fifth column of tiles, row tile s (`y`) and row tile 4 (`z`, in
//   slot 0; the other slots work it out too).
//   A = X X^H, B = b A + c A A: tiles (s, s), (s, s + 1), (s, s + 2) around the corner of five, and (4, 4), (4, 0), (4, 1) in slots
//   0 to 2:
//   all 15 pairs.  X = a X + B X: five row tiles in four slots, and the fifth column in two turns: 28 instructions a step for 25
//   tiles' worth.
// 110592 modes take 1005 to 1046 us, 154 an iteration (108 of matrix instructions, the rest vector instructions and LDS that the two waves of
// a vector unit do not hide); loads and stores alone take 529 us, 3.3 TB/s, as a wave touches 32 bytes of a cache line, and some 240 of them are
// not behind other waves' iterations.
// X, A and B take turns in a wave's 13 KB of LDS, [row][column][mode] with four places of padding a row: rows and columns of a tile are
// read without bank conflicts.  The fifth column of X has a place of its own beside them.
#include "fno_muon_modes.h"

#include <type_traits>

namespace fno {

namespace {

constexpr int kSide = 5, kRows = 4 * kSide, kPitch = 4 * kRows + 4;    // places of a row
constexpr int kWaveModes = 4, kWaves = 4;
constexpr int kPerLaunch = 32;

struct Modes5Entry {
  float2* p;
  const float2* g;
  float2* mom;
  long long modes, si, sj;             // si, sj: distance of rows and columns of X, in values
  unsigned first, skip;                // first block of the launch that belongs to this tensor; blocks of it in earlier launches
  int m, n;
  float keep, move;                    // 1 - lr weight_decay, lr scale
};
struct Modes5List {
  Modes5Entry t[kPerLaunch];
  int count;
  unsigned blocks;
};

__global__ __launch_bounds__(64 * kWaves, 2) void muon_modes5_kernel(Modes5List l, MuonScalars c) {
  __shared__ float2 matrices[kWaves][kRows * kPitch], fifths[kWaves][kRows * 16];
  const unsigned item = (unsigned)xcd_contiguous_item(blockIdx.x, gridDim.x);
  if (item >= l.blocks) return;
  float scale;
  if (!muon_scale(c, scale)) return;
  int k = 0;
  while (k + 1 < l.count && l.t[k + 1].first <= item) ++k;
  const Modes5Entry& t = l.t[k];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 3, md = (lane >> 2) & 3, s = lane >> 4;
  float2 *const S = matrices[w], *const last = fifths[w];              // last: column 16 + j of X, [row][j][mode]
  const long long mode0 = (((long long)(item - t.first) + t.skip) * kWaves + w) * kWaveModes;
  if (mode0 >= t.modes) return;
  const int have = t.modes - mode0 < kWaveModes ? (int)(t.modes - mode0) : kWaveModes;
  const bool here = md < have, here5 = here && 16 + j < t.n;

  // Places: a scalar base for the row and 32 bits of the lane's own.  Lanes past the last mode or column have the last one's values,
  // rows past the last one are its; columns and rows become zeros, which stay zeros, and none of them is stored.
  const unsigned row = (unsigned)t.si, col = (unsigned)t.sj, lane_mode = (unsigned)(here ? md : have - 1);
  const unsigned col5 = (16 + j < t.n ? 16u + j : t.n - 1u) * col + lane_mode;
  const unsigned px = ((4u * s + j) * col + lane_mode) * 8u, py = (col5 + 4u * s * row) * 8u, pz = col5 * 8u;
  auto place = [&](auto* tensor, int r, unsigned own) {
    typedef decltype(tensor) pointer;
    return reinterpret_cast<pointer>((char*)(tensor + mode0 + (long long)r * t.si) + own);
  };
  auto row_of = [&](int r) { return r < 17 || r < t.m ? r : t.m - 1; };
  float2 x[kRows], y[4], z[4];
  {
    float2 ox[kRows], oy[4], oz[4];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      x[i] = *place(t.g, row_of(i), px);
      ox[i] = *place(t.mom, row_of(i), px);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      y[r] = *place(t.g, r, py);
      oy[r] = *place(t.mom, r, py);
      z[r] = *place(t.g, row_of(16 + r), pz);
      oz[r] = *place(t.mom, row_of(16 + r), pz);
    }
    auto step = [&](float2& v, float2& m) { v = make_float2(muon_momentum(c, v.x, m.x), muon_momentum(c, v.y, m.y)); };
    if (scale != 1.0f) {
#pragma unroll
      for (int i = 0; i < kRows; ++i) x[i] = make_float2(x[i].x * scale, x[i].y * scale);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        y[r] = make_float2(y[r].x * scale, y[r].y * scale);
        z[r] = make_float2(z[r].x * scale, z[r].y * scale);
      }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      step(x[i], ox[i]);
      if (here && (i < 17 || i < t.m)) *place(t.mom, i, px) = ox[i];
      if (i >= 17 && i >= t.m) x[i] = make_float2(0.f, 0.f);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      step(y[r], oy[r]);
      step(z[r], oz[r]);
      if (here5) *place(t.mom, r, py) = oy[r];
      if (here5 && s == 0 && (r == 0 || 16 + r < t.m)) *place(t.mom, 16 + r, pz) = oz[r];
      if (16 + j >= t.n) y[r] = make_float2(0.f, 0.f);
      if (16 + j >= t.n || (r > 0 && 16 + r >= t.m)) z[r] = make_float2(0.f, 0.f);
    }
  }
  {
    // |u|^2 in float where that holds its squares, else in double.  The corner tile z counts once.
    auto total = [&](auto zero) {
      decltype(zero) sum = zero, corner = zero;
      auto add = [](auto& to, float2 v) {
        typedef typename std::remove_reference<decltype(to)>::type real;
        to += (real)v.x * (real)v.x;
        to += (real)v.y * (real)v.y;
      };
#pragma unroll
      for (int i = 0; i < kRows; ++i) add(sum, x[i]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        add(sum, y[r]);
        add(corner, z[r]);
      }
      sum += s == 0 ? corner : zero;
      sum += __shfl_xor(sum, 1);
      sum += __shfl_xor(sum, 2);
      sum += __shfl_xor(sum, 16);
      sum += __shfl_xor(sum, 32);
      return sum;
    };
    auto times = [&](auto by) {
      auto one = [&](float2& v) { v = make_float2((float)(v.x * by), (float)(v.y * by)); };
#pragma unroll
      for (int i = 0; i < kRows; ++i) one(x[i]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        one(y[r]);
        one(z[r]);
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

  // The tiles of A and B that this lane's slot works out: (I, J) of turn d, and where their values lie in S
  const int s2 = s + 2 < kSide ? s + 2 : s + 2 - kSide, s4 = s == 1 ? 0 : s == 2 ? 1 : 4;
  const int I[4] = {s, s, s, 4}, J[4] = {s, s + 1, s2, s4};
  auto by_row = [&](int tile) { return (4 * tile + j) * kPitch + md; };          // element (4 tile + j, 0)
  auto by_col = [&](int tile) { return (4 * tile + j) * 4 + md; };               // element (0, 4 tile + j)
  Tile4 q[4];
  auto put = [&]() {
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      if (d == 3 && s == 3) continue;
      float2* const direct = S + 4 * I[d] * kPitch + by_col(J[d]);
      float2* const mirror = S + by_row(J[d]) + 16 * I[d];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        direct[r * kPitch] = make_float2(q[d].r[r], q[d].i[r]);
        if (d == 1 || d == 2 || (d == 3 && s > 0)) mirror[4 * r] = make_float2(q[d].r[r], -q[d].i[r]);
      }
    }
  };

  for (int it = 0; it < c.iterations; ++it) {
    own_fence();
#pragma unroll
    for (int i = 0; i < kRows; ++i) S[i * kPitch + by_col(s)] = x[i];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      S[(4 * s + r) * kPitch + by_col(4)] = y[r];
      last[(4 * s + r) * 16 + 4 * j + md] = y[r];
      if (s == 0) {
        S[(16 + r) * kPitch + by_col(4)] = z[r];
        last[(16 + r) * 16 + 4 * j + md] = z[r];
      }
    }
    own_fence();
    // A(I, J) = sum over columns n of X(I, n) conj X(J, n)
#pragma unroll
    for (int d = 0; d < 4; ++d) clear(q[d]);
    {
      const float2 *p0 = S + by_row(s), *p1 = S + by_row(s + 1), *p2 = S + by_row(s2), *p3 = S + by_row(4), *p4 = S + by_row(s4);
#pragma unroll
      for (int n = 0; n < kRows; ++n) {
        const float2 a = p0[4 * n], b1 = p1[4 * n], b2 = p2[4 * n], a4 = p3[4 * n], b4 = p4[4 * n];
        add_conj_right(q[0], a, a);
        add_conj_right(q[1], a, b1);
        add_conj_right(q[2], a, b2);
        add_conj_right(q[3], a4, b4);
      }
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) q[d].i -= q[d].h;
    own_fence();
    put();
    own_fence();
    // B = b A + c A A, (A A)(I, J) = sum over rows n of conj A(n, I) A(n, J)
#pragma unroll
    for (int d = 0; d < 4; ++d) clear(q[d]);
    {
      const float2 *p0 = S + by_col(s), *p1 = S + by_col(s + 1), *p2 = S + by_col(s2), *p3 = S + by_col(4), *p4 = S + by_col(s4);
#pragma unroll
      for (int n = 0; n < kRows; ++n) {
        const float2 a = p0[n * kPitch], b1 = p1[n * kPitch], b2 = p2[n * kPitch], a4 = p3[n * kPitch], b4 = p4[n * kPitch];
        add_conj_left(q[0], a, a);
        add_conj_left(q[1], a, b1);
        add_conj_left(q[2], a, b2);
        add_conj_left(q[3], a4, b4);
      }
    }
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const float2* const own = S + 4 * I[d] * kPitch + by_col(J[d]);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const float2 v = own[r * kPitch];
        q[d].r[r] = fmaf(c.b, v.x, c.c * q[d].r[r]);
        q[d].i[r] = fmaf(c.b, v.y, c.c * (q[d].i[r] - q[d].h[r]));
        if (d == 0) q[d].r[r] += r == j ? c.a : 0.f;
        if (d == 3) q[d].r[r] += s == 0 && r == j ? c.a : 0.f;
      }
    }
    own_fence();
    put();
    own_fence();
    // X(I, J) = sum over rows n of conj B(n, I) X(n, J)
    Tile4 u[kSide], uy, uz;
#pragma unroll
    for (int T = 0; T < kSide; ++T) clear(u[T]);
    clear(uy);
    clear(uz);
    {
      const float2 *own = S + by_col(s), *tiles = S + by_col(0), *fifth = last + 4 * j + md;
#pragma unroll
      for (int n = 0; n < kRows; ++n) {
        float2 v[kSide];
#pragma unroll
        for (int T = 0; T < kSide; ++T) v[T] = tiles[n * kPitch + 16 * T];
        const float2 vs = own[n * kPitch], f = fifth[n * 16];
        // (here the sign costs less than seven more accumulators)
        const float nx = -x[n].x, nf = -f.x;
#pragma unroll
        for (int T = 0; T < kSide; ++T) {
          u[T].r = mfma4(v[T].x, x[n].x, u[T].r);
          u[T].i = mfma4(v[T].x, x[n].y, u[T].i);
        }
        uy.r = mfma4(vs.x, f.x, uy.r);
        uy.i = mfma4(vs.x, f.y, uy.i);
        uz.r = mfma4(v[4].x, f.x, uz.r);
        uz.i = mfma4(v[4].x, f.y, uz.i);
#pragma unroll
        for (int T = 0; T < kSide; ++T) {
          u[T].r = mfma4(v[T].y, x[n].y, u[T].r);
          u[T].i = mfma4(v[T].y, nx, u[T].i);
        }
        uy.r = mfma4(vs.y, f.y, uy.r);
        uy.i = mfma4(vs.y, nf, uy.i);
        uz.r = mfma4(v[4].y, f.y, uz.r);
        uz.i = mfma4(v[4].y, nf, uz.i);
      }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
#pragma unroll
      for (int T = 0; T < kSide; ++T) x[4 * T + r] = make_float2(u[T].r[r], u[T].i[r]);
      y[r] = make_float2(uy.r[r], uy.i[r]);
      z[r] = make_float2(uz.r[r], uz.i[r]);
    }
  }

  auto moved = [&](float2 p, float2 v) { return make_float2(fmaf(p.x, t.keep, -t.move * v.x), fmaf(p.y, t.keep, -t.move * v.y)); };
  float2 p[kRows], q5[4], q6[4];
#pragma unroll
  for (int i = 0; i < kRows; ++i) p[i] = *place(t.p, row_of(i), px);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    q5[r] = *place(t.p, r, py);
    q6[r] = *place(t.p, row_of(16 + r), pz);
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i)
    if (here && (i < 17 || i < t.m)) *place(t.p, i, px) = moved(p[i], x[i]);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    if (here5) *place(t.p, r, py) = moved(q5[r], y[r]);
    if (here5 && s == 0 && (r == 0 || 16 + r < t.m)) *place(t.p, 16 + r, pz) = moved(q6[r], z[r]);
  }
}

}  // namespace

// us a step of 17 x 17 (20 x 20) for 110592 modes, here and in fno_muon_modes.hip: 935 (1005) and 1513 (1563); for 1536 modes 52 and 57.
// Where a mode's values lie within 4 GB of each other (1.3 million modes of 20 x 20): a lane's place has 32 bits.
bool muon_is_modes5(const MuonTensor& t) {
  return t.modes && t.rows > 16 && t.rows <= 20 && t.cols > 16 && t.cols <= 20 && 20 * (t.cols + 1) * t.batch < (1ll << 29);
}

// Launches of 2^20 blocks at most.
hipError_t launch_muon_modes5(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s) {
  constexpr long long kMost = 1ll << 20;
  Modes5List l;
  l.count = 0;
  l.blocks = 0;
  auto flush = [&]() {
    if (l.count > 0) hipLaunchKernelGGL(muon_modes5_kernel, dim3((l.blocks + 7) / 8 * 8), dim3(64 * kWaves), 0, s, l, c);
    const hipError_t e = l.count > 0 ? hipGetLastError() : hipSuccess;
    l.count = 0;
    l.blocks = 0;
    return e;
  };
  for (int k = 0; k < count; ++k) {
    if (!muon_is_modes5(t[k])) continue;
    const bool tall = t[k].rows > t[k].cols;
    const long long row = (long long)t[k].cols * t[k].batch, column = t[k].batch;
    const long long blocks = (t[k].batch + kWaves * kWaveModes - 1) / (kWaves * kWaveModes);
    for (long long done = 0; done < blocks;) {
      if (l.count == kPerLaunch || l.blocks == kMost) {
        const hipError_t e = flush();
        if (e != hipSuccess) return e;
      }
      const long long here = blocks - done < kMost - l.blocks ? blocks - done : kMost - l.blocks;
      l.t[l.count++] = Modes5Entry{reinterpret_cast<float2*>(t[k].p), reinterpret_cast<const float2*>(t[k].g),
                                   reinterpret_cast<float2*>(t[k].m), (long long)t[k].batch, tall ? column : row, tall ? row : column, l.blocks,
                                   (unsigned)done, tall ? t[k].cols : t[k].rows, tall ? t[k].rows : t[k].cols,
                                   (float)(1.0 - lr * t[k].decay), (float)(lr * t[k].scale)};
      l.blocks += (unsigned)here;
      done += here;
    }
  }
  return flush();
}

}  // namespace fno
