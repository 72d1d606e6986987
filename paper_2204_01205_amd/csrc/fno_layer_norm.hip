// Layer norm with an activation, forward and adjoint: statistics of every point over its channels, fields [B][C][P] (channels
// first, fno_layer_norm_first.hip) or [B][P][C] (channels last, fno_layer_norm_last.hip) in float or bf16.
//
// What the operator moves bounds it: x in and y out (adjoint: x and gy in, gx out), 20 to 40 operations a value.  A point's channels
// fit the registers of a lane, a group of lanes or a block, so every value is read once (but gy of more than 512 channels first); the adjoint works
// the statistics out again from them.  Measured where an elementwise sum of large arrays reaches 5.9 to 6.2 TB/s: forward, 20 channels, 60 x 60 x 64 x 30
// points, 207 us = 5.3 TB/s; adjoint, 20 channels, 128 x 128 x 64 x 32 points, 1545 us = 5.2 TB/s; adjoint of 32768 rows of 1024 in
// bf16, 54 us = 3.7 TB/s.  The gradients of gamma and beta are sums over all points: lanes add up what they see in float over their
// tiles, blocks write their sums, and one more launch adds the blocks' in double, in a fixed order.
#include "fno_layer_norm.h"

namespace fno {

namespace {

constexpr int kColumns = 16, kSlices = 64;

__global__ __launch_bounds__(kColumns * kSlices) void layer_sum_kernel(int C, int blocks, const float* part, float* ggamma, float* gbeta,
                                                                       int add) {
  __shared__ double red[kSlices][kColumns + 1];
  const int j = threadIdx.x % kColumns, slice = threadIdx.x / kColumns, col = blockIdx.x * kColumns + j;
  double s = 0.0;
  if (col < 2 * C) {
#pragma unroll 8
    for (int b = slice; b < blocks; b += kSlices) s += part[(long long)b * 2 * C + col];
  }
  red[slice][j] = s;
  __syncthreads();
  for (int half = kSlices / 2; half >= 1; half /= 2) {
    if (slice < half) red[slice][j] += red[slice + half][j];
    __syncthreads();
  }
  if (slice != 0 || col >= 2 * C) return;
  float* const out = col < C ? ggamma : gbeta;
  const int c = col < C ? col : col - C;
  if (out != nullptr) out[c] = (add ? out[c] : 0.f) + (float)red[0][j];
}

int bwd_blocks(const LayerShape& n) { return n.P == 0 ? 0 : n.last ? layer_last_blocks(n) : layer_first_blocks(n); }

}  // namespace

size_t layer_norm_workspace_bytes(const LayerShape& n) {
  const size_t blocks = (size_t)bwd_blocks(n);
  return (blocks > 0 ? blocks : 1) * 2 * n.C * sizeof(float);
}

hipError_t launch_layer_norm_fwd(const LayerShape& n, const void* x, const float* gamma, const float* beta, void* y, hipStream_t s) {
  const LayerCall a{n, x, nullptr, y, gamma, beta, nullptr};
  return n.last ? launch_layer_last_fwd(a, s) : launch_layer_first_fwd(a, s);
}

hipError_t launch_layer_norm_bwd(const LayerShape& n, const void* x, const float* gamma, const float* beta, const void* gy,
                                 void* gx, float* ggamma, float* gbeta, int accumulate, void* ws, hipStream_t s) {
  const bool sums = ggamma != nullptr || gbeta != nullptr;
  const int blocks = bwd_blocks(n);
  const LayerCall a{n, x, gy, gx, gamma, beta, sums ? static_cast<float*>(ws) : nullptr};
  if (blocks > 0) {
    const hipError_t e = n.last ? launch_layer_last_bwd(a, blocks, s) : launch_layer_first_bwd(a, blocks, s);
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;
  hipLaunchKernelGGL(layer_sum_kernel, dim3((2 * n.C + kColumns - 1) / kColumns), dim3(kColumns * kSlices), 0, s, n.C, blocks,
                     static_cast<const float*>(ws), ggamma, gbeta, accumulate);
  return hipGetLastError();
}

}  // namespace fno
