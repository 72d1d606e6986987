// Layer norm of fields [B][C][P], adjoint.
#include "fno_layer_norm_first.h"

namespace fno {

namespace {

template <class T, int KC, int V, int ACT, bool STREAM>
__global__ __launch_bounds__(kThreads) void first_bwd_kernel(LayerArgs a, long long tiles, const T* x, const T* gy, T* gx) {
  constexpr int LEAST = kLeast<KC>;
  __shared__ float sums[kThreads / 64][2 * KC], affine[2 * KC];
  load_affine(a, affine);
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  float sg[KC], sb[KC];
#pragma unroll
  for (int c = 0; c < KC; ++c) sg[c] = sb[c] = 0.f;
  const long long each = tiles_each<V>(a.P);
  for (long long tile = (long long)blockIdx.x * (kThreads / 64) + w; tile < tiles; tile += (long long)gridDim.x * (kThreads / 64))
    with_tile<T, V>(a, tile, each, [&](auto points, Tile t) {
      constexpr int N = decltype(points)::value;
      const int have = opaque(a.C);
      float xh[KC][N], g[KC][N], off[N], rstd[N], s1[N], s2[N];
      load_channels<T, KC, LEAST, N, STREAM>(a, x, t, have, xh);
      load_channels<T, KC, LEAST, N, STREAM>(a, gy, t, have, g);
      statistics<KC, LEAST, N>(a, have, xh, off, rstd);
#pragma unroll
      for (int u = 0; u < N; ++u) s1[u] = s2[u] = 0.f;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        if (c >= LEAST && c >= have) continue;
        const float ga = affine[c], gk = ga * kArg<ACT>, bk = affine[a.C + c] * kArg<ACT>;
#pragma unroll
        for (int u = 0; u < N; ++u) {
          const float h = (xh[c][u] - off[u]) * rstd[u], gz = g[c][u] * slope_f<ACT>(fmaf(h, gk, bk));
          const bool in = N > 1 || t.mine;
          sb[c] += in ? gz : 0.f;
          sg[c] = in ? fmaf(gz, h, sg[c]) : sg[c];
          xh[c][u] = h;
          g[c][u] = gz * ga;
          s1[u] += g[c][u];
          s2[u] = fmaf(g[c][u], h, s2[u]);
        }
      }
      if (opaque(__builtin_amdgcn_readfirstlane(gx != nullptr)) == 0) return;
      T* to = gx + t.base;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        if (c >= LEAST && c >= have) continue;
#pragma unroll
        for (int u = 0; u < N; ++u) g[c][u] = rstd[u] * (fmaf(-s1[u], a.inv_c, g[c][u]) - xh[c][u] * (s2[u] * a.inv_c));
        store_channel<T, N, STREAM>(to, t, g[c]);
        to += a.P;
      }
    });
  if (a.part == nullptr) return;
#pragma unroll
  for (int c = 0; c < KC; ++c) {
    const float g = wave_sum(sg[c]), b = wave_sum(sb[c]);
    if (lane == 0) {
      sums[w][c] = g;
      sums[w][KC + c] = b;
    }
    __builtin_amdgcn_sched_barrier(0);
  }
  __syncthreads();
  for (int k = threadIdx.x; k < 2 * KC; k += kThreads) {
    const int c = k < KC ? k : k - KC;
    if (c < a.C) a.part[(long long)blockIdx.x * 2 * a.C + (k < KC ? 0 : a.C) + c] = (sums[0][k] + sums[1][k]) + (sums[2][k] + sums[3][k]);
  }
}

// AGAIN: gy is read a second time instead of being kept.  A wave adds a channel's terms over its lanes at once; lane k keeps the
// sums of the wave's channel k.  With 64 channels a wave (more than 512 channels) the 128 registers that 16 waves leave do not hold all: 2 or 3
// are spilled, and 24, 352 bytes a lane, in bf16 with GELU, which costs much (1024 channels, 32768 points: 424 us; f32 184, no activation 145).
template <class T, int K, int V, int ACT, bool STREAM, bool AGAIN>
__global__ __launch_bounds__(1024) void shared_bwd_kernel(LayerArgs a, long long tiles, const T* x, const T* gy, T* gx) {
  extern __shared__ float lds[];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, c0 = w * K, lane = threadIdx.x & 63;
  const int share = a.C - c0 < K ? a.C - c0 : K, stage = waves * 64 * V;
  const float* const affine = lds + 5 * stage + c0;
  load_affine(a, lds + 5 * stage);
  const long long each = tiles_each<V>(a.P), down = (long long)c0 * a.P;
  float sg = 0.f, sb = 0.f;
  for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x)
    with_tile<T, V>(a, tile, each, [&](auto points, Tile t) {
      constexpr int N = decltype(points)::value;
      const int have = opaque(__builtin_amdgcn_readfirstlane(share));
      float xh[K][N], g[AGAIN ? 1 : K][N], off[N], rstd[N], s1[N], s2[N];
      load_channels<T, K, 1, N, STREAM>(a, x + down, t, have, xh);
      if constexpr (!AGAIN) load_channels<T, K, 1, N, STREAM>(a, gy + down, t, have, g);
      shared_statistics<K, N>(a, lds, stage, w, waves, have, xh, off, rstd);
#pragma unroll
      for (int u = 0; u < N; ++u) s1[u] = s2[u] = 0.f;
      const T* from = gy + down;
#pragma unroll
      for (int c = 0; c < K; ++c) {
        if (c >= have) continue;
        const float ga = affine[c], gk = ga * kArg<ACT>, bk = affine[a.C + c] * kArg<ACT>;
        if constexpr (AGAIN) {
          load_channels<T, 1, 1, N, false>(a, from, t, 1, g);
          from += a.P;
        }
        float tg = 0.f, tb = 0.f;
#pragma unroll
        for (int u = 0; u < N; ++u) {
          const float h = (xh[c][u] - off[u]) * rstd[u], gz = g[AGAIN ? 0 : c][u] * slope_f<ACT>(fmaf(h, gk, bk));
          const bool in = N > 1 || t.mine;
          tb += in ? gz : 0.f;
          tg = in ? fmaf(gz, h, tg) : tg;
          xh[c][u] = h;
          const float k = gz * ga;
          if constexpr (!AGAIN) g[c][u] = k;
          s1[u] += k;
          s2[u] = fmaf(k, h, s2[u]);
        }
        tg = wave_sum(tg);
        tb = wave_sum(tb);
        sg += lane == c ? tg : 0.f;
        sb += lane == c ? tb : 0.f;
      }
      put_sums<N>(lds + 3 * stage, w, s1);
      put_sums<N>(lds + 4 * stage, w, s2);
      __syncthreads();
      get_sums<N>(lds + 3 * stage, waves, s1);
      get_sums<N>(lds + 4 * stage, waves, s2);
      if (opaque(__builtin_amdgcn_readfirstlane(gx != nullptr)) == 0) return;
      T* to = gx + down + t.base;
      from = gy + down;
#pragma unroll
      for (int c = 0; c < K; ++c) {
        if (c >= have) continue;
        float o[N];
        if constexpr (AGAIN) {
          const float ga = affine[c], be = affine[a.C + c];
          load_channels<T, 1, 1, N, STREAM>(a, from, t, 1, g);
          from += a.P;
#pragma unroll
          for (int u = 0; u < N; ++u) o[u] = ga * g[0][u] * slope_f<ACT>(fmaf(xh[c][u], ga * kArg<ACT>, be * kArg<ACT>));
        } else {
#pragma unroll
          for (int u = 0; u < N; ++u) o[u] = g[AGAIN ? 0 : c][u];
        }
#pragma unroll
        for (int u = 0; u < N; ++u) o[u] = rstd[u] * (fmaf(-s1[u], a.inv_c, o[u]) - xh[c][u] * (s2[u] * a.inv_c));
        store_channel<T, N, STREAM>(to, t, o);
        to += a.P;
      }
    });
  if (a.part == nullptr || lane >= share) return;
  float* const to = a.part + (long long)blockIdx.x * 2 * a.C + c0 + lane;
  to[0] = sg;
  to[a.C] = sb;
}

// 2048 blocks fill the chip; more where a lane's chain of additions would be longer than 256 tiles (1024 terms of four points a lane).  2^20
// is past any memory.
int blocks_for(long long tiles, int waves) {
  const long long b = (tiles + waves - 1) / waves;
  return (int)std::min(b, std::clamp(b / 256, 2048ll, 1ll << 20));
}

}  // namespace

int layer_first_blocks(const LayerShape& n) {
  int blocks = 0;
  if (is_narrow(n)) {
    with_narrow(n.C, [&](auto kc) {
      constexpr int KC = decltype(kc)::value;
      const int v = n.bf16 ? kBwdPoints<u16, KC, true> : streams(n) ? kBwdPoints<float, KC, true> : kBwdPoints<float, KC, false>;
      blocks = blocks_for(tiles_host(n, v), kThreads / 64);
    });
  } else {
    with_shared(n.C, [&](auto k) { blocks = blocks_for(tiles_host(n, kSharedPoints<decltype(k)::value>), 1); });
  }
  return blocks;
}

hipError_t launch_layer_first_bwd(const LayerCall& c, int blocks, hipStream_t s) {
  const LayerArgs a = layer_args(c);
  return with_layer_kind(c.n, [&](auto t, auto act, auto stream) {
    using T = decltype(t);
    constexpr int ACT = decltype(act)::value;
    constexpr bool S = decltype(stream)::value;
    const T *x = static_cast<const T*>(c.x), *gy = static_cast<const T*>(c.gy);
    T* const gx = static_cast<T*>(c.out);
    if (is_narrow(c.n)) {
      with_narrow(a.C, [&](auto kc) {
        constexpr int KC = decltype(kc)::value, V = kBwdPoints<T, KC, S>;
        hipLaunchKernelGGL((first_bwd_kernel<T, KC, V, ACT, S>), dim3(blocks), dim3(kThreads), 0, s, a, tiles_host(c.n, V), x, gy, gx);
      });
    } else {
      with_shared(a.C, [&](auto k) {
        constexpr int K = decltype(k)::value, V = kSharedPoints<K>;
        const int waves = (a.C + K - 1) / K;
        hipLaunchKernelGGL((shared_bwd_kernel<T, K, V, ACT, S, K == 64>), dim3(blocks), dim3(64 * waves), 
                           (5 * waves * 64 * V + 2 * a.C) * sizeof(float), s,
                           a, tiles_host(c.n, V), x, gy, gx);
      });
    }
  });
}

}  // namespace fno
