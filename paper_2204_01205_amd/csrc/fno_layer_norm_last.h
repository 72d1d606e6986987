// Layer norm of rows: fields [B][P][C], channels last.
//
// Up to some 400 channels (512 that are no whole 16-byte pieces) a wave takes a tile of rows, a stretch of memory that starts at a
// multiple of 16 bytes whatever C is: it goes to LDS in 16-byte pieces, a group of G lanes (a power of two) takes a row, E = 4 .. 8
// channels each, and the results go the same way back.  A wave's LDS is its own, so waves need no barrier.  More channels: a row a wave
// or a block, in registers, straight from memory.
#pragma once
#include "fno_layer_norm.h"

namespace fno {

namespace {

// ------------------------------------------------------------------------------------------ tiles of rows

// LDS accesses of a wave are worked in order; this keeps the compiler to it.
__device__ __forceinline__ void wave_fence() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}
template <class T> constexpr int kPasses = sizeof(T) == 4 ? 4 : 8;       // rows of a lane group in a tile, at most

struct Rows {
  long long rows;
  int lg;                    // G = 2^lg lanes a row
  int each;                  // rows of a tile
};
// A tile's values between memory and LDS: E pieces a lane (at most kPasses rows of C <= E G channels for each of 64 / G groups).  Pieces past
// the end read the last one again, so that no load waits behind a branch.
template <int E, bool STREAM, class T>
__device__ __forceinline__ void tile_in(const T* from, T* to, int count) {
  constexpr int V = kVec<T>;
  const int lane = threadIdx.x & 63, whole = count / V;
  if (whole > 0) {
    pack<T> q[E];
#pragma unroll
    for (int u = 0; u < E; ++u) q[u] = load_pack<STREAM>(from + (unsigned)min(u * 64 + lane, whole - 1) * V);
#pragma unroll
    for (int u = 0; u < E; ++u) *reinterpret_cast<pack<T>*>(to + min(u * 64 + lane, whole - 1) * V) = q[u];
  }
  if (whole * V + lane < count) to[whole * V + lane] = from[whole * V + lane];
}
template <int E, bool STREAM, class T>
__device__ __forceinline__ void tile_out(const T* from, T* to, int count) {
  constexpr int V = kVec<T>;
  const int lane = threadIdx.x & 63, whole = count / V;
#pragma unroll
  for (int u = 0; u < E; ++u)
    if (u * 64 + lane < whole) store_pack<STREAM>(to + (unsigned)(u * 64 + lane) * V, *reinterpret_cast<const pack<T>*>(from + (u * 64 + lane) * V));
  if (whole * V + lane < count) to[whole * V + lane] = from[whole * V + lane];
}
// E values of a row in LDS, `have` of them this lane's.  ALIGNED: they start at a multiple of their length, or of 16 bytes.
template <int E, bool ALIGNED, class T>
__device__ __forceinline__ void lds_read(const T* p, int have, float (&v)[E]) {
  if constexpr (ALIGNED && sizeof(T) == 4) {
#pragma unroll
    for (int u = 0; u < E; u += 4) {
      const v4f q = *reinterpret_cast<const v4f*>(p + u);
#pragma unroll
      for (int k = 0; k < 4; ++k) v[u + k] = q[k];
    }
  } else if constexpr (ALIGNED && E == 8) {
    unpack(*reinterpret_cast<const u32x4*>(p), v);
  } else {
#pragma unroll
    for (int u = 0; u < E; ++u) v[u] = load1(p + (u < have ? u : 0));
  }
}
template <int E, bool ALIGNED, class T>
__device__ __forceinline__ void lds_write(T* p, int have, const float (&v)[E]) {
  if constexpr (ALIGNED && sizeof(T) == 4) {
    if (have > 0)
#pragma unroll
      for (int u = 0; u < E; u += 4) *reinterpret_cast<v4f*>(p + u) = v4f{v[u], v[u + 1], v[u + 2], v[u + 3]};
  } else if constexpr (ALIGNED && E == 8) {
    if (have > 0) *reinterpret_cast<u32x4*>(p) = repack(v);
  } else {
#pragma unroll
    for (int u = 0; u < E; ++u)
      if (u < have) store1(p + u, v[u]);
  }
}
// x becomes xh
template <int E, bool ALIGNED>
__device__ __forceinline__ float row_statistics(const LayerArgs& a, int lg, int have, float (&x)[E]) {
  float s = 0.f, o = 0.f, q = 0.f;
#pragma unroll
  for (int u = 0; u < E; ++u) s += ALIGNED || u < have ? x[u] : 0.f;
  const float about = lanes_sum(s, lg) * a.inv_c;
#pragma unroll
  for (int u = 0; u < E; ++u) {
    x[u] = ALIGNED || u < have ? x[u] - about : 0.f;
    o += x[u];
    q = fmaf(x[u], x[u], q);
  }
  const float off = lanes_sum(o, lg) * a.inv_c, rstd = rstd_of(a, off, lanes_sum(q, lg));
#pragma unroll
  for (int u = 0; u < E; ++u) x[u] = (x[u] - off) * rstd;
  return rstd;
}

// ------------------------------------------------------------------------------------------ a row a wave or a block

// Sums over the W waves of a row; red: 2 W floats, another pair of them for every stage
template <int W>
__device__ __forceinline__ void row_sum2(float& s, float& q, float* red) {
  s = wave_sum(s);
  q = wave_sum(q);
  if constexpr (W > 1) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
      red[2 * w] = s;
      red[2 * w + 1] = q;
    }
    __syncthreads();
    s = q = 0.f;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      s += red[2 * k];
      q += red[2 * k + 1];
    }
  }
}
// x becomes xh.  A lane's piece k is channels [(k L + l) V, ...), L lanes a row.
template <int W, int N, int V>
__device__ __forceinline__ float wide_statistics(const LayerArgs& a, int left, float (&x)[N][V], float* red) {
  constexpr int STEP = 64 * W * V;
  float s = 0.f, q = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int u = 0; u < V; ++u) s += x[k][u];                // zeros past the end
  row_sum2<W>(s, q, red);
  const float about = s * a.inv_c;
  s = q = 0.f;
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int u = 0; u < V; ++u) {
      x[k][u] = k * STEP + u < left ? x[k][u] - about : 0.f;
      s += x[k][u];
      q = fmaf(x[k][u], x[k][u], q);
    }
  row_sum2<W>(s, q, red + 2 * W);
  const float off = s * a.inv_c, rstd = rstd_of(a, off, q);
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int u = 0; u < V; ++u) x[k][u] = (x[k][u] - off) * rstd;
  return rstd;
}

// W == 1: a block of four waves has four rows.
template <int W> constexpr int kRowThreads = W == 1 ? 256 : 64 * W;
// ------------------------------------------------------------------------------------------ launches

inline int lanes_of(int C) {
  int lg = 0;
  while ((C + (1 << lg) - 1) >> lg > 8) ++lg;
  return lg;
}
// Channels of a lane; whether its share of a row is whole 16-byte pieces
template <int SIZE, class F>
void with_channels(int C, F&& f) {
  const int lg = lanes_of(C), e = (C + (1 << lg) - 1) >> lg;
  const bool whole = C == e << lg && (e * SIZE) % 16 == 0;
  if (e == 8 && whole) f(std::integral_constant<int, 8>(), std::true_type());
  else if (e <= 4 && SIZE == 4 && whole && e == 4) {
    if constexpr (SIZE == 4) f(std::integral_constant<int, 4>(), std::true_type());
  } else if (e <= 4) f(std::integral_constant<int, 4>(), std::false_type());
  else if (e == 5) f(std::integral_constant<int, 5>(), std::false_type());
  else if (e == 6) f(std::integral_constant<int, 6>(), std::false_type());
  else if (e == 7) f(std::integral_constant<int, 7>(), std::false_type());
  else f(std::integral_constant<int, 8>(), std::false_type());
}
// Waves of a row and 16-byte pieces of a lane: two or four of them, whose sums are the less work the fewer waves have a row (16384 rows
// of 1024 in bf16, adjoint: 33.6 us with one, 102 with four), as far as the registers go (8192 rows of 8192 in bf16, adjoint: 308 us with
// four waves, 204 with sixteen).
template <int SIZE, bool BWD, class F>
void with_row(int C, F&& f) {
  const int pieces = (C * SIZE + 1023) / 1024;             // of a wave
  if (pieces <= 2) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 2>());
  if (pieces <= 4) return f(std::integral_constant<int, 1>(), std::integral_constant<int, 4>());
  if (pieces <= 8) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 2>());
  if constexpr (!(BWD && SIZE == 2))
    if (pieces <= 16) return f(std::integral_constant<int, 4>(), std::integral_constant<int, 4>());
  if (pieces <= 32) return f(std::integral_constant<int, 16>(), std::integral_constant<int, 2>());
  if constexpr (SIZE == 4) f(std::integral_constant<int, 16>(), std::integral_constant<int, 4>());
}
inline int size_of(const LayerShape& n) { return n.bf16 ? 2 : 4; }
// Rows that are wide enough go without LDS, in bf16 where they are whole 16-byte pieces.  us for 65536 rows, forward and adjoint, in
// tiles against registers: f32 of 512 50 and 101 against 42 and 93, of 300 30 and 59 against 33 and 64; bf16 of 512 37 and 83 against
// 37 and 69, of 448 34 and 86 against 41 and 78, of 511 42 and 97 against 51 and 120.
inline bool in_tiles(const LayerShape& n) { return n.C < (n.bf16 ? 480 : 384) || (n.bf16 && n.C <= 512 && n.C % 8 != 0); }
// Tiles start at multiples of 16 bytes.  They are as long as kPasses allows where that makes 2048 of them, eight waves a compute
// unit, else shorter: 53760 rows of 27 in bf16 take 6.6 us, 8.9 with 420 tiles.
inline Rows rows_of(const LayerShape& n) {
  Rows r{n.B * n.P, lanes_of(n.C), 0};
  int passes = n.bf16 ? kPasses<u16> : kPasses<float>;
  const int group = 64 >> r.lg;
  while (passes > 1 && group * (passes / 2) * n.C * size_of(n) % 16 == 0 && r.rows < 2048ll * group * passes) passes /= 2;
  r.each = group * passes;
  return r;
}
inline long long row_tiles(const LayerShape& n) {
  const Rows r = rows_of(n);
  return (r.rows + r.each - 1) / r.each;
}
// A wave's tile is at most 64 lanes by 8 channels in each of its passes.
static_assert(2 * 4 * 64 * 8 * kPasses<float> * sizeof(float) <= 65536 && 2 * 4 * 64 * 8 * kPasses<u16> * sizeof(u16) <= 65536,
              "the adjoint's two tiles of four waves stay within what a block has without asking");
inline size_t tile_bytes(const LayerShape& n) { return (size_t)4 * rows_of(n).each * n.C * size_of(n); }      // of a block's four waves

}  // namespace

}  // namespace fno
