// What the Muon step's kernels share.
#pragma once
#include "fno_device.h"

namespace fno {

// Numbers of a step that all matrices have in common
struct MuonScalars {
  float mu, a, b, c, max_norm;
  int nesterov, iterations;
  double eps;
  const float* norm;      // device scalar, nullable
};

// Steps of the spectral weights: two (fno_muon_modes2.hip) or five tiles of four channels on either side (fno_muon_modes5.hip), and
// all others (fno_muon_modes.hip)
bool muon_is_modes2(const MuonTensor& t);
hipError_t launch_muon_modes2(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s);
bool muon_is_modes5(const MuonTensor& t);
hipError_t launch_muon_modes5(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s);
hipError_t launch_muon_modes(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s);

// Steps of the small real matrices of a list (fno_muon_small.hip)
bool muon_is_small(const MuonTensor& t);
hipError_t launch_muon_small(const MuonTensor* t, int count, const MuonScalars& c, double lr, hipStream_t s);

// Steps of the other real matrices (fno_muon_dense.hip)
size_t muon_dense_bytes(const MuonTensor* t, int count);
hipError_t launch_muon_dense(const MuonTensor* t, int count, const MuonScalars& c, double lr, void* ws, hipStream_t s);

namespace {

// What the gradient is multiplied by; false where the norm is not finite.
__device__ __forceinline__ bool muon_scale(const MuonScalars& c, float& scale) {
  scale = 1.0f;
  if (c.norm == nullptr) return true;
  const float norm = *c.norm;
  if (!(norm <= 3.402823466e38f)) return false;
  if (norm > c.max_norm) scale = c.max_norm / norm;
  return true;
}
// New momentum, and what is made orthogonal
__device__ __forceinline__ float muon_momentum(const MuonScalars& c, float g, float& m) {
  m = fmaf(c.mu, m, g);
  return c.nesterov ? fmaf(c.mu, m, g) : m;
}
// 1 / (|u|_F + eps); a matrix of zeros stays one, one with an infinity becomes NaN as a whole.  Squares are in double, which
// holds those of all floats.
__device__ __forceinline__ double muon_inverse(double squares, double eps) {
  return squares == 0.0 ? 0.0 : squares < __builtin_huge_val() ? 1.0 / (sqrt(squares) + eps) : __builtin_nan("");
}

}  // namespace

}  // namespace fno
