// What layer norm's kernels share: accesses, statistics, and the sums of the gradients of gamma and beta.
#pragma once
#include "fno_norm_device.h"
#include <algorithm>

namespace fno {

// One call.  Blocks of the adjoint write their share of the sums over points to part, [block][ggamma, gbeta][C].
struct LayerCall {
  LayerShape n;
  const void *x, *gy;        // gy: adjoint only
  void* out;                 // y, or gx (nullable)
  const float *gamma, *beta;
  float* part;               // null: the sums are not asked for
};
// Blocks of the adjoint.
int layer_first_blocks(const LayerShape& n);
int layer_last_blocks(const LayerShape& n);
hipError_t launch_layer_first_fwd(const LayerCall& a, hipStream_t s);
hipError_t launch_layer_first_bwd(const LayerCall& a, int blocks, hipStream_t s);
hipError_t launch_layer_last_fwd(const LayerCall& a, hipStream_t s);
hipError_t launch_layer_last_bwd(const LayerCall& a, int blocks, hipStream_t s);

namespace {

struct LayerArgs {
  int B, C;
  long long P;
  float inv_c, eps;
  const float *gamma, *beta;
  float* part;
};

// V values at an address aligned to one of them
template <int BYTES> struct piece_of;
template <> struct piece_of<2> { typedef u16 type; };
template <> struct piece_of<4> { typedef unsigned type; };
template <> struct piece_of<8> { typedef unsigned type __attribute__((ext_vector_type(2))); };
template <> struct piece_of<16> { typedef u32x4 type; };
template <int V, bool STREAM>
__device__ __forceinline__ void load_values(const float* p, float (&v)[V]) {
#pragma unroll
  for (int u = 0; u < V; u += 4) load_run<(V < 4 ? V : 4), STREAM>(p + u, v + u);
}
template <int V, bool STREAM>
__device__ __forceinline__ void store_values(float* p, const float (&v)[V]) {
#pragma unroll
  for (int u = 0; u < V; u += 4) store_run<(V < 4 ? V : 4), STREAM>(p + u, v + u);
}
template <int V, bool STREAM>
__device__ __forceinline__ void load_values(const u16* p, float (&v)[V]) {
  typedef typename piece_of<2 * V>::type vec;
  typedef vec loose __attribute__((aligned(2)));
  vec q;
  if constexpr (STREAM) q = __builtin_nontemporal_load(reinterpret_cast<const loose*>(p));
  else q = *reinterpret_cast<const loose*>(p);
  if constexpr (V == 1) v[0] = bf16_low(q);
  else if constexpr (V == 2) {
    v[0] = bf16_low(q);
    v[1] = bf16_high(q);
  } else {
#pragma unroll
    for (int u = 0; u < V / 2; ++u) {
      v[2 * u] = bf16_low(q[u]);
      v[2 * u + 1] = bf16_high(q[u]);
    }
  }
}
template <int V, bool STREAM>
__device__ __forceinline__ void store_values(u16* p, const float (&v)[V]) {
  typedef typename piece_of<2 * V>::type vec;
  typedef vec loose __attribute__((aligned(2)));
  vec q;
  if constexpr (V == 1) q = (u16)bf16_pair(v[0], 0.f);
  else if constexpr (V == 2) q = bf16_pair(v[0], v[1]);
  else {
#pragma unroll
    for (int u = 0; u < V / 2; ++u) q[u] = bf16_pair(v[2 * u], v[2 * u + 1]);
  }
  if constexpr (STREAM) __builtin_nontemporal_store(q, reinterpret_cast<loose*>(p));
  else *reinterpret_cast<loose*>(p) = q;
}
// `count` of them, zeros behind
template <int V, bool STREAM, class T>
__device__ __forceinline__ void load_some(const T* p, int count, float (&v)[V]) {
  if (count >= V) {
    load_values<V, STREAM>(p, v);
  } else {
#pragma unroll
    for (int u = 0; u < V; ++u) v[u] = u < count ? load1(p + u) : 0.f;
  }
}
template <int V, bool STREAM, class T>
__device__ __forceinline__ void store_some(T* p, int count, const float (&v)[V]) {
  if (count >= V) {
    store_values<V, STREAM>(p, v);
  } else {
#pragma unroll
    for (int u = 0; u < V; ++u)
      if (u < count) store1(p + u, v[u]);
  }
}

// Statistics of a point in two sweeps over registers.  about = sum x / C is the mean up to its rounding; with d = x - about, which is
// exact near it, the mean is about + off with off = sum d / C, and the variance sum d^2 / C - off^2, from which next to nothing is
// subtracted.  Where all channels are the same, far from zero, that difference is rounding of either sign: with eps it counts as eps at
// least (a comparison, so that a NaN stays one).  xh = (d - off) rstd.
__device__ __forceinline__ float rstd_of(const LayerArgs& a, float off, float squares) {
  const float sum = fmaf(squares, a.inv_c, fmaf(-off, off, a.eps)), var = sum < a.eps ? a.eps : sum;
  const float r = __builtin_amdgcn_rsqf(var);
  // one Newton step: the instruction is off by an ulp.  An infinite r (a variance of zero) stays one, and so does a NaN.
  const float e = fmaf(-var * r, r, 1.0f);
  const float better = fmaf(0.5f * r, e, r);
  return r < 3e38f ? better : r;
}

template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, ROWS, 0xF, true));
}
// Sums over groups of 2^lg lanes, in every lane
__device__ __forceinline__ float lanes_sum(float v, int lg) {
  if (lg > 0) v = dpp_add<0xB1>(v);        // lane ^ 1
  if (lg > 1) v = dpp_add<0x4E>(v);        // lane ^ 2
  if (lg > 2) v = dpp_add<0x141>(v);       // mirrored in eights
  if (lg > 3) v = dpp_add<0x140>(v);       // mirrored in rows of 16
  if (lg > 4) v += __shfl_xor(v, 16);
  if (lg > 5) v += __shfl_xor(v, 32);
  return v;
}
__device__ __forceinline__ float wave_sum(float v) { return lanes_sum(v, 6); }

// out of the memory-side cache's reach: the nontemporal hint
inline bool streams(const LayerShape& n) { return (double)n.B * n.C * (double)n.P * (n.bf16 ? 2 : 4) > (double)kStreamBytes; }
template <class F>
hipError_t with_layer_kind(const LayerShape& n, F&& f) {
  auto stream = [&](auto t, auto act) {
    if (streams(n)) f(t, act, std::true_type());
    else f(t, act, std::false_type());
  };
  auto act = [&](auto t) {
    if (n.act == 0) stream(t, std::integral_constant<int, 0>());
    else if (n.act == 1) stream(t, std::integral_constant<int, 1>());
    else stream(t, std::integral_constant<int, 2>());
  };
  if (n.bf16) act(u16());
  else act(float());
  return hipGetLastError();
}
inline LayerArgs layer_args(const LayerCall& a) {
  return LayerArgs{a.n.B, a.n.C, (long long)a.n.P, 1.0f / (float)a.n.C, (float)a.n.eps, a.gamma, a.beta, a.part};
}

}  // namespace

}  // namespace fno
