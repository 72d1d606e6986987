// Layer norm of fields [B][C][P], forward.
#include "fno_layer_norm_first.h"

namespace fno {

namespace {

template <class T, int KC, int V, int ACT, bool STREAM>
__global__ __launch_bounds__(kThreads) void first_fwd_kernel(LayerArgs a, long long tiles, const T* x, T* y) {
  constexpr int LEAST = kLeast<KC>;
  __shared__ float affine[2 * KC];
  load_affine(a, affine);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const long long each = tiles_each<V>(a.P);
  for (long long tile = (long long)blockIdx.x * (kThreads / 64) + w; tile < tiles; tile += (long long)gridDim.x * (kThreads / 64))
    with_tile<T, V>(a, tile, each, [&](auto points, Tile t) {
      constexpr int N = decltype(points)::value;
      const int have = opaque(a.C);
      float v[KC][N], off[N], rstd[N];
      load_channels<T, KC, LEAST, N, STREAM>(a, x, t, have, v);
      statistics<KC, LEAST, N>(a, have, v, off, rstd);
      T* to = y + t.base;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        if (c >= LEAST && c >= have) continue;
        const float ga = affine[c], be = affine[a.C + c];
#pragma unroll
        for (int u = 0; u < N; ++u) v[c][u] = act_f<ACT>(fmaf((v[c][u] - off[u]) * rstd[u], ga, be));
        store_channel<T, N, STREAM>(to, t, v[c]);
        to += a.P;
      }
    });
}

template <class T, int K, int V, int ACT, bool STREAM>
__global__ __launch_bounds__(1024) void shared_fwd_kernel(LayerArgs a, long long tiles, const T* x, T* y) {
  extern __shared__ float lds[];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, c0 = w * K;
  const int share = a.C - c0 < K ? a.C - c0 : K, stage = waves * 64 * V;
  const float* const affine = lds + 3 * stage + c0;
  load_affine(a, lds + 3 * stage);
  const long long each = tiles_each<V>(a.P), down = (long long)c0 * a.P;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x)
    with_tile<T, V>(a, tile, each, [&](auto points, Tile t) {
      constexpr int N = decltype(points)::value;
      const int have = opaque(__builtin_amdgcn_readfirstlane(share));
      float v[K][N], off[N], rstd[N];
      load_channels<T, K, 1, N, STREAM>(a, x + down, t, have, v);
      shared_statistics<K, N>(a, lds, stage, w, waves, have, v, off, rstd);
      T* to = y + down + t.base;
#pragma unroll
      for (int c = 0; c < K; ++c) {
        if (c >= have) continue;
        const float ga = affine[c], be = affine[a.C + c];
#pragma unroll
        for (int u = 0; u < N; ++u) v[c][u] = act_f<ACT>(fmaf((v[c][u] - off[u]) * rstd[u], ga, be));
        store_channel<T, N, STREAM>(to, t, v[c]);
        to += a.P;
      }
    });
}

unsigned grid_of(long long blocks) { return (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20); }

}  // namespace

hipError_t launch_layer_first_fwd(const LayerCall& c, hipStream_t s) {
  return with_layer_kind(c.n, [&](auto t, auto act, auto stream) {
    using T = decltype(t);
    constexpr int ACT = decltype(act)::value;
    constexpr bool S = decltype(stream)::value;
    const LayerArgs a = layer_args(c);
    const T* const x = static_cast<const T*>(c.x);
    T* const y = static_cast<T*>(c.out);
    if (is_narrow(c.n)) {
      with_narrow(a.C, [&](auto kc) {
        constexpr int KC = decltype(kc)::value, V = kFwdPoints<T, KC>;
        const long long tiles = tiles_host(c.n, V);
        hipLaunchKernelGGL((first_fwd_kernel<T, KC, V, ACT, S>), dim3(grid_of((tiles + 3) / 4)), dim3(kThreads), 0, s, a, tiles, x, y);
      });
    } else {
      with_shared(a.C, [&](auto k) {
        constexpr int K = decltype(k)::value, V = kSharedPoints<K>;
        const int waves = (a.C + K - 1) / K;
        const long long tiles = tiles_host(c.n, V);
        hipLaunchKernelGGL((shared_fwd_kernel<T, K, V, ACT, S>), dim3(grid_of(tiles)), dim3(64 * waves),
                           (3 * waves * 64 * V + 2 * a.C) * sizeof(float),
                           s, a, tiles, x, y);
      });
    }
  });
}

}  // namespace fno
