// Layer norm of fields [B][C][P]: a lane has V consecutive points.  Up to 12 channels, and up to 24 of
// many points, all of a point's are in one lane's registers and waves need nothing of each other; else they are dealt to the waves of a
// block, which exchange their sums through LDS.
#pragma once
#include "fno_layer_norm.h"

namespace fno {

namespace {

// Tiles of 64 V points of one batch entry.  The last of an entry goes in tiles of 64, a point a lane.
struct Tile {
  long long base;            // its first point in channel 0: the same in all lanes
  unsigned at;               // from there to this lane's first point, in bytes; past the entry's end, its last one
  bool mine;                 // not past the end
};
template <int V>
__device__ __forceinline__ long long tiles_each(long long P) { return (P + 64 * V - 1) / (64 * V); }
// A value that the compiler takes for a new one: it makes a copy of a loop for every uniform condition that does not change in it,
// sixteen of these for four conditions.
template <class V>
__device__ __forceinline__ V opaque(V v) {
  asm volatile("" : "+s"(v));
  return v;
}
// a scalar base and 32 bits of a lane's own, which is an address of the instructions
template <class T>
__device__ __forceinline__ T* place(T* base, const Tile& t) {
  typedef typename std::conditional<std::is_const<T>::value, const char, char>::type byte;
  return reinterpret_cast<T*>(reinterpret_cast<byte*>(base) + t.at);
}
// a value that is the same in all lanes, in scalar registers (a division leaves it in a vector register)
__device__ __forceinline__ long long uniform(long long v) {
  const unsigned lo = __builtin_amdgcn_readfirstlane((int)v), hi = __builtin_amdgcn_readfirstlane((int)(v >> 32));
  return (long long)((unsigned long long)hi << 32 | lo);
}
// body(std::integral_constant<int, V or 1>, tile) for tile number `tile` of all entries
template <class T, int V, class F>
__device__ __forceinline__ void with_tile(const LayerArgs& a, long long tile, long long each, F&& body) {
  const long long b = uniform(a.B == 1 ? 0 : tile / each), p = (tile - b * each) * (64 * V), base = b * a.C * a.P + p;
  const int lane = threadIdx.x & 63;
  asm volatile("" ::: "memory");       // gamma and beta stay in LDS: kept for all tiles they would take 60 registers of 20 channels
  if (a.P - p >= 64 * V) {
    body(std::integral_constant<int, V>(), Tile{base, (unsigned)(lane * V * sizeof(T)), true});
  } else {
    const int left = (int)(a.P - p);
    for (int k = 0; k < left; k += 64) body(std::integral_constant<int, 1>(), Tile{base + k, (unsigned)(min(lane, left - 1 - k) * sizeof(T)), k + lane < left});
  }
}
// V values of K channels; channels from `have` on read the last one again and count for nothing.  LEAST: have is at least that.
// A channel's place is the one before's and P more: K products with P would be kept in more scalar registers than there are.
template <class T, int K, int LEAST, int V, bool STREAM>
__device__ __forceinline__ void load_channels(const LayerArgs& a, const T* x, const Tile& t, int have, float (&v)[K][V]) {
  const T* from = x + t.base;
#pragma unroll
  for (int c = 0; c < K; ++c) {
    load_values<V, STREAM && (V > 1)>(place(from, t), v[c]);
    if (c + 1 < LEAST || c + 1 < have) from += a.P;
  }
}
template <class T, int V, bool STREAM>
__device__ __forceinline__ void store_channel(T* to, const Tile& t, const float (&v)[V]) {
  if constexpr (V == 1) {
    if (t.mine) store1(place(to, t), v[0]);
  } else {
    store_values<V, STREAM>(place(to, t), v);
  }
}
// x becomes x - about; off and rstd of every point
template <int K, int LEAST, int V>
__device__ __forceinline__ void statistics(const LayerArgs& a, int have, float (&x)[K][V], float (&off)[V], float (&rstd)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float s = 0.f, o = 0.f, q = 0.f;
#pragma unroll
    for (int c = 0; c < K; ++c) s += c < LEAST || c < have ? x[c][v] : 0.f;
    const float about = s * a.inv_c;
#pragma unroll
    for (int c = 0; c < K; ++c) {
      const float d = x[c][v] - about, in = c < LEAST || c < have ? d : 0.f;
      o += in;
      q = fmaf(in, in, q);
      x[c][v] = d;
    }
    off[v] = o * a.inv_c;
    rstd[v] = rstd_of(a, off[v], q);
  }
}
// gamma and beta of a block's channels, ones and zeros where there are none, to LDS: [2][C], in a kernel's first lines
__device__ __forceinline__ void load_affine(const LayerArgs& a, float* affine) {
  for (int c = threadIdx.x; c < a.C; c += blockDim.x) {
    affine[c] = a.gamma ? a.gamma[c] : 1.f;
    affine[a.C + c] = a.beta ? a.beta[c] : 0.f;
  }
  __syncthreads();
}

// A block's waves take K channels each of the same tile.  Sums go through LDS, [stage][wave][point]; the stages lie apart, so
// that a stage's barrier also says that the one before the last has been read.
template <int V>
__device__ __forceinline__ void put_sums(float* lds, int w, const float (&s)[V]) {
#pragma unroll
  for (int u = 0; u < V; ++u) lds[w * (64 * V) + u * 64 + (threadIdx.x & 63)] = s[u];
}
template <int V>
__device__ __forceinline__ void get_sums(const float* lds, int waves, float (&s)[V]) {
#pragma unroll
  for (int u = 0; u < V; ++u) s[u] = 0.f;
  for (int k = 0; k < waves; ++k)
#pragma unroll
    for (int u = 0; u < V; ++u) s[u] += lds[k * (64 * V) + u * 64 + (threadIdx.x & 63)];
}
// stage: floats of one
template <int K, int V>
__device__ __forceinline__ void shared_statistics(const LayerArgs& a, float* lds, int stage, int w, int waves, int have, float (&x)[K][V],
                                                  float (&off)[V], float (&rstd)[V]) {
  float s[V], q[V];
#pragma unroll
  for (int u = 0; u < V; ++u) {
    s[u] = 0.f;
#pragma unroll
    for (int c = 0; c < K; ++c) s[u] += c < have ? x[c][u] : 0.f;
  }
  put_sums<V>(lds, w, s);
  __syncthreads();
  get_sums<V>(lds, waves, s);
#pragma unroll
  for (int u = 0; u < V; ++u) {
    const float about = s[u] * a.inv_c;
    s[u] = q[u] = 0.f;
#pragma unroll
    for (int c = 0; c < K; ++c) {
      const float d = x[c][u] - about;
      s[u] += c < have ? d : 0.f;
      q[u] = c < have ? fmaf(d, d, q[u]) : q[u];
      x[c][u] = d;
    }
  }
  put_sums<V>(lds + stage, w, s);
  put_sums<V>(lds + 2 * stage, w, q);
  __syncthreads();
  get_sums<V>(lds + stage, waves, s);
  get_sums<V>(lds + 2 * stage, waves, q);
#pragma unroll
  for (int u = 0; u < V; ++u) {
    off[u] = s[u] * a.inv_c;
    rstd[u] = rstd_of(a, off[u], q[u]);
  }
}

// All channels of a point in a lane's registers: up to 12 always, up to 24 where there are points enough to hide a lane's chain over
// them.  us, forward and adjoint, a lane's own against shared: 24 channels in f32 at 2^17 points 9.3 and 16.4 against 7.0 and 15.9,
// bf16 at 2^18 8.4 and 18.7 against 8.9 and 20.3, 20 channels in f32 at 2^24 542 and 752 against 500 and 958; 32 channels at 2^21 133
// and 268 against 84 and 195.
constexpr long long kEnoughPoints = 1ll << 18;
inline bool is_narrow(const LayerShape& n) { return n.C <= 12 || (n.C <= 24 && n.B * n.P >= kEnoughPoints); }
// Points of a lane: what leaves registers for enough waves.  us: bf16 forward, 16 channels, 2^21 points 26.9 with two, 30.4 with four; f32,
// 8 channels, 23.5 with four, 26.8 with two.  Adjoint: bf16, 16 channels, 50.6 with two, 89.9 with four; f32, 20 channels, 112 with
// one, 127 with two, 165 with four, but out of the caches (128 x 128 x 64 x 32 points) 1544 with two, 1600 with one.
template <class T, int KC> constexpr int kFwdPoints = sizeof(T) == 4 || KC <= 8 ? 4 : 2;
template <class T, int KC, bool STREAM> constexpr int kBwdPoints = KC <= 8 ? 4 : sizeof(T) == 4 && KC >= 16 && !STREAM ? 1 : 2;
// Of a lane that shares its points: 64 channels, bf16, 2^19 points, us forward and adjoint 28 and 63 with two, 38 and 78 with one.
template <int K> constexpr int kSharedPoints = K <= 16 ? 2 : 1;

// Channels of a lane, and how many of them there are at least
template <int KC> constexpr int kLeast = KC == 8 ? 1 : KC - 3;
template <class F>
void with_narrow(int C, F&& f) {
  if (C <= 8) f(std::integral_constant<int, 8>());
  else if (C <= 12) f(std::integral_constant<int, 12>());
  else if (C <= 16) f(std::integral_constant<int, 16>());
  else if (C <= 20) f(std::integral_constant<int, 20>());
  else f(std::integral_constant<int, 24>());
}
// Channels of a wave, so that there are at most 16 waves
template <class F>
void with_shared(int C, F&& f) {
  if (C <= 128) f(std::integral_constant<int, 8>());
  else if (C <= 256) f(std::integral_constant<int, 16>());
  else if (C <= 512) f(std::integral_constant<int, 32>());
  else f(std::integral_constant<int, 64>());
}
inline long long tiles_host(const LayerShape& n, int V) { return n.B * ((n.P + 64 * V - 1) / (64 * V)); }

}  // namespace

}  // namespace fno
