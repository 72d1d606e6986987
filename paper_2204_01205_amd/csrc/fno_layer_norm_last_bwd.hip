// Layer norm of rows, adjoint.
#include "fno_layer_norm_last.h"

namespace fno {

namespace {

template <class T, int E, bool ALIGNED, int ACT, bool STREAM>
__global__ __launch_bounds__(kThreads) void tile_bwd_kernel(LayerArgs a, Rows r, const T* x, const T* gy, T* gx) {
  extern __shared__ __align__(16) char mem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = r.each, group = lane >> r.lg, first = (lane & ((1 << r.lg) - 1)) * E;
  const int have = a.C - first < 0 ? 0 : a.C - first < E ? a.C - first : E;
  T *const mine = reinterpret_cast<T*>(mem) + (size_t)w * 2 * rows * a.C, *const cot = mine + rows * a.C;
  float ga[E], be[E], sg[E], sb[E];
#pragma unroll
  for (int u = 0; u < E; ++u) {
    ga[u] = u < have && a.gamma ? a.gamma[first + u] : 1.f;
    be[u] = (u < have && a.beta ? a.beta[first + u] : 0.f) * kArg<ACT>;
    sg[u] = sb[u] = 0.f;
  }
  const long long tiles = (r.rows + rows - 1) / rows;
  for (long long tile = (long long)blockIdx.x * (kThreads / 64) + w; tile < tiles; tile += (long long)gridDim.x * (kThreads / 64)) {
    const long long row0 = tile * rows;
    const int count = (int)(r.rows - row0 < rows ? r.rows - row0 : rows);
    tile_in<E, STREAM>(x + row0 * a.C, mine, count * a.C);
    tile_in<E, STREAM>(gy + row0 * a.C, cot, count * a.C);
    wave_fence();
#pragma unroll 1
    for (int row = group; row < count; row += 64 >> r.lg) {
      const int at = row * a.C + (have > 0 ? first : 0);
      float v[E], g[E], s1 = 0.f, s2 = 0.f;
      lds_read<E, ALIGNED>(mine + at, have, v);
      lds_read<E, ALIGNED>(cot + at, have, g);
      const float rstd = row_statistics<E, ALIGNED>(a, r.lg, have, v);
#pragma unroll
      for (int u = 0; u < E; ++u) {
        const float gz = ALIGNED || u < have ? g[u] * slope_f<ACT>(fmaf(v[u], ga[u] * kArg<ACT>, be[u])) : 0.f;
        sb[u] += gz;
        sg[u] = ALIGNED || u < have ? fmaf(gz, v[u], sg[u]) : 0.f;
        g[u] = gz * ga[u];
        s1 += g[u];
        s2 = ALIGNED || u < have ? fmaf(g[u], v[u], s2) : s2;
      }
      s1 = lanes_sum(s1, r.lg) * a.inv_c;
      s2 = lanes_sum(s2, r.lg) * a.inv_c;
#pragma unroll
      for (int u = 0; u < E; ++u) g[u] = rstd * ((g[u] - s1) - v[u] * s2);
      lds_write<E, ALIGNED>(cot + at, have, g);
    }
    wave_fence();
    if (gx != nullptr) tile_out<E, STREAM>(cot, gx + row0 * a.C, count * a.C);
    wave_fence();
  }
  if (a.part == nullptr) return;
  // the sums of a channel: over the lanes that have it, then over the waves
  __syncthreads();
  float* const sums = reinterpret_cast<float*>(mem);       // [wave][ggamma, gbeta][C]
#pragma unroll
  for (int u = 0; u < E; ++u) {
    float g = sg[u], b = sb[u];
    for (int off = 1 << r.lg; off < 64; off <<= 1) {
      g += __shfl_xor(g, off);
      b += __shfl_xor(b, off);
    }
    if (lane < (1 << r.lg) && u < have) {
      sums[w * 2 * a.C + first + u] = g;
      sums[w * 2 * a.C + a.C + first + u] = b;
    }
  }
  __syncthreads();
  for (int k = threadIdx.x; k < 2 * a.C; k += kThreads)
    a.part[(long long)blockIdx.x * 2 * a.C + k] = (sums[k] + sums[2 * a.C + k]) + (sums[4 * a.C + k] + sums[6 * a.C + k]);
}

// With sixteen waves a row (f32 from 8193 channels, bf16 from 4097 on) 128 registers do not hold all: 2 are spilled, and with an activation 24 to
// 34, 100 to 140 bytes a lane (4096 rows of 16384, GELU against none: f32 259 and 211 us, bf16 170 and 136).
template <class T, int W, int N, int ACT, bool STREAM>
__global__ __launch_bounds__(kRowThreads<W>) void wide_bwd_kernel(LayerArgs a, long long rows, const T* x, const T* gy, T* gx) {
  constexpr int V = kVec<T>, STEP = 64 * W * V, PER = W == 1 ? 4 : 1;
  __shared__ float red[W == 1 ? 1 : 6 * W];
  const int l = W == 1 ? threadIdx.x & 63 : threadIdx.x, first = l * V, left = a.C - first;
  const int w = W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  float sg[N][V], sb[N][V];
#pragma unroll
  for (int k = 0; k < N; ++k)
#pragma unroll
    for (int u = 0; u < V; ++u) sg[k][u] = sb[k][u] = 0.f;
  for (long long row = (long long)blockIdx.x * PER + w; row < rows; row += (long long)gridDim.x * PER) {
    const long long at = row * a.C + first;
    float v[N][V], g[N][V], s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      load_some<V, STREAM>(x + at + k * STEP, left - k * STEP, v[k]);
      load_some<V, STREAM>(gy + at + k * STEP, left - k * STEP, g[k]);
    }
    const float rstd = wide_statistics<W, N, V>(a, left, v, red);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float ga[V], be[V];
#pragma unroll
      for (int u = 0; u < V; ++u) {
        ga[u] = 1.f;
        be[u] = 0.f;
      }
      if (a.gamma) load_some<V, false>(a.gamma + first + k * STEP, left - k * STEP, ga);
      if (a.beta && ACT != 0) load_some<V, false>(a.beta + first + k * STEP, left - k * STEP, be);
#pragma unroll
      for (int u = 0; u < V; ++u) {
        const float gz = g[k][u] * slope_f<ACT>(fmaf(v[k][u], ga[u], be[u]) * kArg<ACT>);
        if (k * STEP + u < left) {
          sb[k][u] += gz;
          sg[k][u] = fmaf(gz, v[k][u], sg[k][u]);
          g[k][u] = gz * ga[u];
          s1 += g[k][u];
          s2 = fmaf(g[k][u], v[k][u], s2);
        }
      }
    }
    row_sum2<W>(s1, s2, red + 4 * W);
    s1 *= a.inv_c;
    s2 *= a.inv_c;
    if (gx == nullptr) continue;
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
      for (int u = 0; u < V; ++u) g[k][u] = rstd * ((g[k][u] - s1) - v[k][u] * s2);
      store_some<V, STREAM>(gx + at + k * STEP, left - k * STEP, g[k]);
    }
  }
  if (a.part == nullptr) return;
  float* const to = a.part + (long long)blockIdx.x * 2 * a.C + first;
  if constexpr (W == 1) {              // the four waves' sums one after the other: [ggamma, gbeta][C]
    extern __shared__ float sums[];
    for (int turn = 0; turn < 4; ++turn) {
      if (turn > 0) __syncthreads();
      if (turn != w) continue;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        float og[V], ob[V];
#pragma unroll
        for (int u = 0; u < V; ++u) og[u] = ob[u] = 0.f;
        if (turn > 0) {
          load_some<V, false>(sums + first + k * STEP, left - k * STEP, og);
          load_some<V, false>(sums + a.C + first + k * STEP, left - k * STEP, ob);
        }
#pragma unroll
        for (int u = 0; u < V; ++u) {
          sg[k][u] += og[u];
          sb[k][u] += ob[u];
        }
        if (turn < 3) {
          store_some<V, false>(sums + first + k * STEP, left - k * STEP, sg[k]);
          store_some<V, false>(sums + a.C + first + k * STEP, left - k * STEP, sb[k]);
        }
      }
    }
    if (w != 3) return;
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    store_some<V, false>(to + k * STEP, left - k * STEP, sg[k]);
    store_some<V, false>(to + a.C + k * STEP, left - k * STEP, sb[k]);
  }
}

// ------------------------------------------------------------------------------------------ launches

// `most` blocks, more where a lane's chain of additions would be longer than 256 rows or tiles (2048 terms of eight rows a tile); 2^20 is past
// any memory.
int blocks_for(long long items, int each, int most) {
  const long long b = (items + each - 1) / each;
  return (int)std::min(b, std::clamp(b / 256, (long long)most, 1ll << 20));
}

}  // namespace

int layer_last_blocks(const LayerShape& n) {
  if (in_tiles(n)) return blocks_for(row_tiles(n), 4, 1024);
  int blocks = 0;
  auto count = [&](auto w, auto) {
    constexpr int W = decltype(w)::value;
    blocks = W == 1 ? blocks_for(n.B * n.P, 4, 1024) : blocks_for(n.B * n.P, 1, W == 4 ? 1024 : 512);
  };
  if (n.bf16) with_row<2, true>(n.C, count);
  else with_row<4, true>(n.C, count);
  return blocks;
}

hipError_t launch_layer_last_bwd(const LayerCall& c, int blocks, hipStream_t s) {
  return with_layer_kind(c.n, [&](auto t, auto act, auto stream) {
    using T = decltype(t);
    constexpr int ACT = decltype(act)::value;
    constexpr bool S = decltype(stream)::value;
    const LayerArgs a = layer_args(c);
    const T *x = static_cast<const T*>(c.x), *gy = static_cast<const T*>(c.gy);
    T* const gx = static_cast<T*>(c.out);
    const long long rows = a.B * a.P;
    if (in_tiles(c.n)) {
      with_channels<sizeof(T)>(a.C, [&](auto e, auto whole) {
          const size_t sums = (size_t)8 * a.C * sizeof(float), bytes = 2 * tile_bytes(c.n) > sums ? 2 * tile_bytes(c.n) : sums;
          hipLaunchKernelGGL((tile_bwd_kernel<T, decltype(e)::value, decltype(whole)::value, ACT, S>), dim3(blocks), dim3(kThreads), bytes, s, a,
                             rows_of(c.n), x, gy, gx);
      });
    } else {
      with_row<sizeof(T), true>(a.C, [&](auto w, auto n) {
        constexpr int W = decltype(w)::value;
        hipLaunchKernelGGL((wide_bwd_kernel<T, W, decltype(n)::value, ACT, S>), dim3(blocks), dim3(kRowThreads<W>),
                           W == 1 ? 2 * a.C * sizeof(float) : 0, s, a, rows, x, gy, gx);
      });
    }
  });
}

}  // namespace fno
