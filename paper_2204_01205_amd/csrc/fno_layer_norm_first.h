// Layer norm of fields [B][C][P]: a lane has V consecutive points.  Up to 32 channels all of a point's are in one lane's registers
// and waves need nothing of each other; more are dealt to the waves of a block, which exchange their sums through LDS.
#pragma once
#include "fno_layer_norm.h"

namespace fno {

namespace {

// Tiles of 64 V points of one batch entry.  The last of an entry goes in tiles of 64, a point a lane.
struct Tile {
  long long at;              // this lane's first point, in channel 0
  int left;                  // points of the entry from there on, V at most
};
template <int V>
__device__ __forceinline__ long long tiles_each(long long P) { return (P + 64 * V - 1) / (64 * V); }
// body(std::integral_constant<int, V or 1>, tile) for tile number `tile` of all entries
template <int V, class F>
__device__ __forceinline__ void with_tile(const LayerArgs& a, long long tile, long long each, F&& body) {
  const long long b = tile / each, p = (tile - b * each) * (64 * V), base = b * a.C * a.P + p;
  const int lane = threadIdx.x & 63;
  if (a.P - p >= 64 * V) {
    body(std::integral_constant<int, V>(), Tile{base + lane * V, V});
  } else {
    const int left = (int)(a.P - p);
    for (int k = 0; k < left; k += 64) body(std::integral_constant<int, 1>(), Tile{base + k + lane, k + lane < left ? 1 : 0});
  }
}
// V values of K channels; channels from `have` on read that one's again and count for nothing
template <class T, int K, int V, bool STREAM>
__device__ __forceinline__ void load_channels(const LayerArgs& a, const T* x, const Tile& t, int have, float (&v)[K][V]) {
#pragma unroll
  for (int c = 0; c < K; ++c) {
    const T* const from = x + t.at + (long long)(c < have ? c : have - 1) * a.P;
    if constexpr (V == 1) v[c][0] = t.left > 0 ? load1(from) : 0.f;
    else load_values<V, STREAM>(from, v[c]);
  }
}
template <class T, int V, bool STREAM>
__device__ __forceinline__ void store_channel(T* to, const Tile& t, const float (&v)[V]) {
  if constexpr (V == 1) {
    if (t.left > 0) store1(to, v[0]);
  } else {
    store_values<V, STREAM>(to, v);
  }
}
// x becomes x - about; off and rstd of every point
template <int K, int V>
__device__ __forceinline__ void statistics(const LayerArgs& a, float (&x)[K][V], float (&off)[V], float (&rstd)[V]) {
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float s = 0.f, o = 0.f, q = 0.f;
#pragma unroll
    for (int c = 0; c < K; ++c) s += c < a.C ? x[c][v] : 0.f;
    const float about = s * a.inv_c;
#pragma unroll
    for (int c = 0; c < K; ++c) {
      const float d = x[c][v] - about;
      o += c < a.C ? d : 0.f;
      q = c < a.C ? fmaf(d, d, q) : q;
      x[c][v] = d;
    }
    off[v] = o * a.inv_c;
    rstd[v] = rstd_of(a, off[v], q);
  }
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

constexpr int kNarrow = 32;
// Points of a lane: as many registers as leave three or four waves a SIMD.
template <class T, int KC> constexpr int kFwdPoints = 4;
template <class T, int KC> constexpr int kBwdPoints = sizeof(T) == 4 ? (KC <= 8 ? 4 : 2) : (KC <= 16 ? 4 : 2);
template <int K> constexpr int kSharedPoints = K <= 16 ? 2 : 1;

template <class F>
void with_narrow(int C, F&& f) {
  if (C <= 8) f(std::integral_constant<int, 8>());
  else if (C <= 12) f(std::integral_constant<int, 12>());
  else if (C <= 16) f(std::integral_constant<int, 16>());
  else if (C <= 20) f(std::integral_constant<int, 20>());
  else if (C <= 24) f(std::integral_constant<int, 24>());
  else f(std::integral_constant<int, 32>());
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
