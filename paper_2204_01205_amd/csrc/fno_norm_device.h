// What group norm and layer norm share: accesses of 16 bytes in float or bf16, activations and their slopes.
#pragma once
#include "fno_device.h"

#include <type_traits>

namespace fno {

namespace {

typedef unsigned short u16;
template <class T> constexpr int kVec = 16 / (int)sizeof(T);      // values of a 16-byte access

__device__ __forceinline__ float load1(const float* p) { return *p; }
__device__ __forceinline__ float load1(const u16* p) { return bf16_low(*p); }
__device__ __forceinline__ void store1(float* p, float v) { *p = v; }
__device__ __forceinline__ void store1(u16* p, float v) { *p = (u16)bf16_pair(v, 0.f); }

// 16 bytes at an aligned address, and the values in them
template <class T> struct pack_of;
template <> struct pack_of<float> { typedef v4f type; };
template <> struct pack_of<u16> { typedef u32x4 type; };
template <class T> using pack = typename pack_of<T>::type;
template <bool STREAM, class T>
__device__ __forceinline__ pack<T> load_pack(const T* p) { return ld_once<STREAM>(reinterpret_cast<const pack<T>*>(p)); }
template <bool STREAM, class T>
__device__ __forceinline__ void store_pack(T* p, pack<T> v) { st_once<STREAM>(reinterpret_cast<pack<T>*>(p), v); }
__device__ __forceinline__ void unpack(v4f q, float (&v)[4]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) v[u] = q[u];
}
__device__ __forceinline__ void unpack(u32x4 q, float (&v)[8]) {
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    v[2 * u] = bf16_low(q[u]);
    v[2 * u + 1] = bf16_high(q[u]);
  }
}
__device__ __forceinline__ v4f repack(const float (&v)[4]) { return v4f{v[0], v[1], v[2], v[3]}; }
__device__ __forceinline__ u32x4 repack(const float (&v)[8]) {
  return u32x4{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
}

// exp(-z) as a power of two; for z below -88 it is infinite and the sigmoid zero, as in the definition
__device__ __forceinline__ float sigmoid_f(float z) {
  return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504089f));
}
template <int ACT>
__device__ __forceinline__ float act_f(float z) {
  if constexpr (ACT == 1) return gelu_fast_f(z);
  if constexpr (ACT == 2) return z * sigmoid_f(z);
  return z;
}
// act'(z) of z / kArg<ACT>.  GELU: Phi + z phi with both from one exponential, by the upper tail exp(-z^2 / 2) t P(t) of
// gelu_and_grad_f; with z in units of sqrt(2 / log2 e) the exponent is a plain square.  With G = 1 + e (z phi(0) - t P) at |z|
// it is G right of zero and 1 - G left of it.
template <int ACT> constexpr float kArg = ACT == 1 ? 0.84932180028f : 1.0f;        // sqrt(log2(e) / 2)
template <int ACT>
__device__ __forceinline__ float slope_f(float z) {
  if constexpr (ACT == 1) {
    const float a = fabsf(z), t = __builtin_amdgcn_rcpf(fmaf(a, 0.4f / kArg<1>, 1.0f));
    float q = fmaf(t, 5.5231631e-02f, -2.5018391e-01f);
    q = fmaf(t, q, 3.3274594e-01f);
    q = fmaf(t, q, 1.8495135e-02f);
    q = fmaf(t, q, 1.8670905e-01f);
    q = fmaf(t, q, 1.5700214e-01f);
    const float e = __builtin_amdgcn_exp2f(-z * z);
    const float w = e * fmaf(-t, q, a * (0.39894228040f / kArg<1>));
    return z < 0.f ? -w : 1.0f + w;
  }
  if constexpr (ACT == 2) {
    const float s = sigmoid_f(z);
    return s * fmaf(z, 1.0f - s, 1.0f);
  }
  return 1.0f;
}

}  // namespace

}  // namespace fno
