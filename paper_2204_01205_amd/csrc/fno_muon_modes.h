// What the Muon step's kernels for spectral weights share: complex 4 x 4 tiles of many modes at a time.
#pragma once
#include "fno_muon.h"

namespace fno {

namespace {

__device__ __forceinline__ v4f mfma4(float a, float b, v4f c) { return __builtin_amdgcn_mfma_f32_4x4x1f32(a, b, c, 0, 0, 0); }
// LDS accesses of a wave are worked in order; this keeps the compiler to it.
__device__ __forceinline__ void own_fence() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}
// A complex tile.  In sums with a conjugate the imaginary part is i - h: an operand's sign would take an instruction a step.
struct Tile4 {
  v4f r, i, h;
};
__device__ __forceinline__ void clear(Tile4& t) { t.r = t.i = t.h = v4f{0.f, 0.f, 0.f, 0.f}; }
// t += a conj b
__device__ __forceinline__ void add_conj_right(Tile4& t, float2 a, float2 b) {
  t.r = mfma4(a.x, b.x, t.r);
  t.i = mfma4(a.y, b.x, t.i);
  t.h = mfma4(a.x, b.y, t.h);
  t.r = mfma4(a.y, b.y, t.r);
}
// t += conj a b
__device__ __forceinline__ void add_conj_left(Tile4& t, float2 a, float2 b) {
  t.r = mfma4(a.x, b.x, t.r);
  t.i = mfma4(a.x, b.y, t.i);
  t.h = mfma4(a.y, b.x, t.h);
  t.r = mfma4(a.y, b.y, t.r);
}

}  // namespace

}  // namespace fno
