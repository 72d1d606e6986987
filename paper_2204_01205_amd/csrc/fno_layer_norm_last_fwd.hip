// Layer norm of rows, forward.
#include "fno_layer_norm_last.h"

namespace fno {

namespace {

template <class T, int E, bool ALIGNED, int ACT, bool STREAM>
__global__ __launch_bounds__(kThreads) void tile_fwd_kernel(LayerArgs a, Rows r, const T* x, T* y) {
  extern __shared__ __align__(16) char mem[];
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = r.each, group = lane >> r.lg, first = (lane & ((1 << r.lg) - 1)) * E;
  const int have = a.C - first < 0 ? 0 : a.C - first < E ? a.C - first : E;
  T* const mine = reinterpret_cast<T*>(mem) + (size_t)w * rows * a.C;
  float ga[E], be[E];
#pragma unroll
  for (int u = 0; u < E; ++u) {
    ga[u] = u < have && a.gamma ? a.gamma[first + u] : 1.f;
    be[u] = u < have && a.beta ? a.beta[first + u] : 0.f;
  }
  const long long tiles = (r.rows + rows - 1) / rows;
  for (long long tile = (long long)blockIdx.x * (kThreads / 64) + w; tile < tiles; tile += (long long)gridDim.x * (kThreads / 64)) {
    const long long row0 = tile * rows;
    const int count = (int)(r.rows - row0 < rows ? r.rows - row0 : rows);
    tile_in<E, STREAM>(x + row0 * a.C, mine, count * a.C);
    wave_fence();
#pragma unroll 1
    for (int row = group; row < count; row += 64 >> r.lg) {      // lanes of a group go through it together
      T* const at = mine + row * a.C + (have > 0 ? first : 0);
      float v[E];
      lds_read<E, ALIGNED>(at, have, v);
      row_statistics<E, ALIGNED>(a, r.lg, have, v);
#pragma unroll
      for (int u = 0; u < E; ++u) v[u] = act_f<ACT>(fmaf(v[u], ga[u], be[u]));
      lds_write<E, ALIGNED>(at, have, v);
    }
    wave_fence();
    tile_out<E, STREAM>(mine, y + row0 * a.C, count * a.C);
    wave_fence();
  }
}

template <class T, int W, int N, int ACT, bool STREAM>
__global__ __launch_bounds__(kRowThreads<W>) void wide_fwd_kernel(LayerArgs a, long long rows, const T* x, T* y) {
  constexpr int V = kVec<T>, STEP = 64 * W * V, PER = W == 1 ? 4 : 1;
  __shared__ float red[W == 1 ? 1 : 4 * W];
  const int l = W == 1 ? threadIdx.x & 63 : threadIdx.x, first = l * V, left = a.C - first;
  for (long long row = (long long)blockIdx.x * PER + (W == 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0); row < rows;
       row += (long long)gridDim.x * PER) {
    const T* const from = x + row * a.C + first;
    T* const to = y + row * a.C + first;
    float v[N][V];
#pragma unroll
    for (int k = 0; k < N; ++k) load_some<V, STREAM>(from + k * STEP, left - k * STEP, v[k]);
    wide_statistics<W, N, V>(a, left, v, red);
#pragma unroll
    for (int k = 0; k < N; ++k) {
      float ga[V], be[V];
#pragma unroll
      for (int u = 0; u < V; ++u) {
        ga[u] = 1.f;
        be[u] = 0.f;
      }
      if (a.gamma) load_some<V, false>(a.gamma + first + k * STEP, left - k * STEP, ga);
      if (a.beta) load_some<V, false>(a.beta + first + k * STEP, left - k * STEP, be);
#pragma unroll
      for (int u = 0; u < V; ++u) v[k][u] = act_f<ACT>(fmaf(v[k][u], ga[u], be[u]));
      store_some<V, STREAM>(to + k * STEP, left - k * STEP, v[k]);
    }
  }
}

unsigned grid_of(long long blocks) { return (unsigned)(blocks < (1 << 20) ? blocks : 1 << 20); }

}  // namespace

hipError_t launch_layer_last_fwd(const LayerCall& c, hipStream_t s) {
  return with_layer_kind(c.n, [&](auto t, auto act, auto stream) {
    using T = decltype(t);
    constexpr int ACT = decltype(act)::value;
    constexpr bool S = decltype(stream)::value;
    const LayerArgs a = layer_args(c);
    const T* const x = static_cast<const T*>(c.x);
    T* const y = static_cast<T*>(c.out);
    const long long rows = a.B * a.P;
    if (in_tiles(c.n)) {
      with_channels<sizeof(T)>(a.C, [&](auto e, auto whole) {
        hipLaunchKernelGGL((tile_fwd_kernel<T, decltype(e)::value, decltype(whole)::value, ACT, S>), dim3(grid_of((row_tiles(c.n) + 3) / 4)),
                             dim3(kThreads), tile_bytes(c.n), s, a, rows_of(c.n), x, y);
      });
    } else {
      with_row<sizeof(T), false>(a.C, [&](auto w, auto n) {
        constexpr int W = decltype(w)::value;
        hipLaunchKernelGGL((wide_fwd_kernel<T, W, decltype(n)::value, ACT, S>), dim3(grid_of(W == 1 ? (rows + 3) / 4 : rows)),
                           dim3(kRowThreads<W>), 0, s, a, rows, x, y);
      });
    }
  });
}

}  // namespace fno
