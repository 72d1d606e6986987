// One AdamW step over the tensors of a list with moments in 32 or 8 bits, the norm of their gradients, and what 8-bit
// moments stand for.
#include "fno_device.h"

namespace fno {

namespace {

typedef unsigned char u8;
typedef unsigned short u16;
typedef u8 v4u8 __attribute__((ext_vector_type(4)));

constexpr int kGroup = 256;            // values that share an exponent
constexpr int kPerLaunch = 64;         // tensors whose addresses go with one launch's arguments (3.5 KB)
constexpr long long kPiece = 4096;     // values that a block takes: of one tensor

struct AdamwEntry {
  float* p;
  const float* g;
  void *m, *v;
  u8* e;
  long long n;
  unsigned first;      // first piece of the launch that belongs to this tensor
  float keep;          // 1 - lr weight_decay
};
struct AdamwList {
  AdamwEntry t[kPerLaunch];
  int count, base;     // tensors of this launch; place of the first one in the caller's list
};
struct AdamwScalars {
  float beta1, omb1, beta2, omb2, eps, lr1, ic2, max_norm;   // lr1 = lr / (1 - beta1^t), ic2 = 1 / (1 - beta2^t)
  unsigned key;        // of the rounding's random bits: seed and step
  const float* norm;
};

// the tensor that a piece belongs to: the last one that starts at or before it
__device__ __forceinline__ int tensor_of(const AdamwList& l, unsigned piece) {
  int lo = 0, hi = l.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (l.t[mid].first <= piece) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__host__ __device__ __forceinline__ unsigned mix_bits(unsigned x) {
  x ^= x >> 16;
  x *= 0xCB4F2D3Bu;
  x ^= x >> 13;
  x *= 0xFDB6A5C3u;
  return x ^ (x >> 16);
}

// What the gradient is multiplied by; false where the norm is not finite.
__device__ __forceinline__ bool clip_scale(const AdamwScalars& c, float& scale) {
  scale = 1.0f;
  if (c.norm == nullptr) return true;
  const float norm = *c.norm;
  if (!(norm <= 3.402823466e38f)) return false;
  if (norm > c.max_norm) scale = c.max_norm / norm;
  return true;
}

// The moments, each product and sum rounded by itself: with 8-bit codes the random rounding then sees the same value as
// any other 32-bit evaluation in this order.
__device__ __forceinline__ void moments(const AdamwScalars& c, float g, float& m, float& v) {
#pragma clang fp contract(off)
  const float a = c.beta1 * m, b = c.omb1 * g;
  m = a + b;
  const float gg = g * g;
  const float d = c.beta2 * v, e = c.omb2 * gg;
  v = d + e;
}
__device__ __forceinline__ float updated(const AdamwScalars& c, float keep, float p, float m, float v) {
  return p * keep - c.lr1 * m / (sqrtf(v * c.ic2) + c.eps);
}

__global__ __launch_bounds__(kThreads) void adamw32_kernel(AdamwList l, AdamwScalars c) {
  const AdamwEntry& t = l.t[tensor_of(l, blockIdx.x)];
  float scale;
  if (!clip_scale(c, scale)) return;
  const long long at = (long long)(blockIdx.x - t.first) * kPiece;
  const long long end = at + kPiece < t.n ? at + kPiece : t.n;
  float *m = static_cast<float*>(t.m), *v = static_cast<float*>(t.v);
  for (long long i = at + threadIdx.x; i < end; i += kThreads) {
    float mi = m[i], vi = v[i];
    moments(c, t.g[i] * scale, mi, vi);
    m[i] = mi;
    v[i] = vi;
    t.p[i] = updated(c, t.keep, t.p[i], mi, vi);
  }
}

// ---- 8-bit moments.  With the bits of a float >> 20 (exponent and three bits), a code is their distance from those of
// the smallest power, and rounding up or down at random is adding 20 random bits before the shift.

constexpr int kSpanM = 15, kSpanV = 31;      // powers of two below the shared one

// Shared exponent for the largest of the absolute values' bits: rounded up to four significant bits, so that no code
// rounds past the last one; 255 where a value is not finite.
__device__ __forceinline__ unsigned shared_exponent(unsigned top, unsigned span) {
  if (top >= 0x7F800000u) return 255u;
  const unsigned e = (top + 0xFFFFFu) >> 23;
  return min(max(e, span + 1u), 254u);
}
__device__ __forceinline__ unsigned encode_m(float x, unsigned e, unsigned r) {
  const unsigned bits = __builtin_bit_cast(unsigned, x) & 0x7FFFFFFFu, low = (e - kSpanM) << 3, first = ((low + 1u) << 20);
  unsigned code;
  if (bits >= first) code = min(((bits + (r << 4)) >> 20) - low, 127u);
  else code = __builtin_bit_cast(float, first) * ((float)r * (1.0f / 65536.0f)) < fabsf(x) ? 1u : 0u;
  return x < 0.f ? code + 128u : code;
}
__device__ __forceinline__ unsigned encode_v(float x, unsigned e, unsigned r) {
  const unsigned bits = __builtin_bit_cast(unsigned, x), low = (e - kSpanV) << 3;
  const int code = (int)((bits + (r << 4)) >> 20) - (int)low;
  return bits == 0u ? 0u : (unsigned)min(max(code, 1), 255);
}
__device__ __forceinline__ float decode_m(unsigned code, unsigned e) {
  const unsigned mag = code & 127u;
  const unsigned bits = e == 255u ? 0x7FC00000u : mag == 0u ? 0u : (mag << 20) + ((e - kSpanM) << 23);
  return __builtin_bit_cast(float, bits | ((code & 128u) << 24));
}
__device__ __forceinline__ float decode_v(unsigned code, unsigned e) {
  const unsigned bits = e == 255u ? 0x7FC00000u : code == 0u ? 0u : (code << 20) + ((e - kSpanV) << 23);
  return __builtin_bit_cast(float, bits);
}
__device__ __forceinline__ unsigned wave_max(unsigned v) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v = max(v, (unsigned)__shfl_xor((int)v, off));
  return v;
}

// A wave takes one block of 256 values at a time, four to a lane.
__global__ __launch_bounds__(kThreads) void adamw8_kernel(AdamwList l, AdamwScalars c) {
  const int k = tensor_of(l, blockIdx.x);
  const AdamwEntry& t = l.t[k];
  float scale;
  if (!clip_scale(c, scale)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const unsigned key = mix_bits(c.key ^ (unsigned)(l.base + k));
  const long long first = (long long)(blockIdx.x - t.first) * (kPiece / kGroup), blocks = (t.n + kGroup - 1) / kGroup;
  u8 *m = static_cast<u8*>(t.m), *v = static_cast<u8*>(t.v);
  for (long long q = first + wave; q < first + kPiece / kGroup && q < blocks; q += kThreads / 64) {
    const unsigned em = t.e[2 * q], ev = t.e[2 * q + 1];
    const unsigned block = mix_bits(mix_bits((unsigned)q + key) + (unsigned)(q >> 32));
    float mi[4], vi[4];
    unsigned top_m = 0, top_v = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = q * kGroup + 4 * lane + u;
      mi[u] = 0.f;
      vi[u] = 0.f;
      if (i < t.n) {
        mi[u] = decode_m(m[i], em);
        vi[u] = decode_v(v[i], ev);
        moments(c, t.g[i] * scale, mi[u], vi[u]);
        t.p[i] = updated(c, t.keep, t.p[i], mi[u], vi[u]);
      }
      top_m = max(top_m, __builtin_bit_cast(unsigned, mi[u]) & 0x7FFFFFFFu);
      top_v = max(top_v, __builtin_bit_cast(unsigned, vi[u]) & 0x7FFFFFFFu);
    }
    const unsigned nm = shared_exponent(wave_max(top_m), kSpanM), nv = shared_exponent(wave_max(top_v), kSpanV);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = q * kGroup + 4 * lane + u;
      const unsigned r = mix_bits(block + (unsigned)(4 * lane + u) * 0x9E3779B1u);
      if (i < t.n) {
        m[i] = nm == 255u ? 0 : (u8)encode_m(mi[u], nm, r & 0xFFFFu);
        v[i] = nv == 255u ? 0 : (u8)encode_v(vi[u], nv, r >> 16);
      }
    }
    if (lane == 0) { t.e[2 * q] = (u8)nm; t.e[2 * q + 1] = (u8)nv; }
  }
}

// p and g of an entry hold the outputs here
__global__ __launch_bounds__(kThreads) void adamw_read_kernel(AdamwList l) {
  const AdamwEntry& t = l.t[tensor_of(l, blockIdx.x)];
  const long long at = (long long)(blockIdx.x - t.first) * kPiece;
  const long long end = at + kPiece < t.n ? at + kPiece : t.n;
  const u8 *m = static_cast<const u8*>(t.m), *v = static_cast<const u8*>(t.v);
  u16 *mo = reinterpret_cast<u16*>(t.p), *vo = reinterpret_cast<u16*>(const_cast<float*>(t.g));
  for (long long i = at + threadIdx.x; i < end; i += kThreads) {
    const long long q = i / kGroup;
    mo[i] = (u16)(__builtin_bit_cast(unsigned, decode_m(m[i], t.e[2 * q])) >> 16);
    vo[i] = (u16)(__builtin_bit_cast(unsigned, decode_v(v[i], t.e[2 * q + 1])) >> 16);
  }
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < kThreads / 64; ++w) s += red[w];
  return s;
}

__global__ __launch_bounds__(kThreads) void grad_norm_partial_kernel(AdamwList l, double* part) {
  __shared__ double red[kThreads / 64];
  const AdamwEntry& t = l.t[tensor_of(l, blockIdx.x)];
  const long long at = (long long)(blockIdx.x - t.first) * kPiece;
  const long long end = at + kPiece < t.n ? at + kPiece : t.n;
  double s = 0.0;
  for (long long i = at + threadIdx.x; i < end; i += kThreads) s += (double)t.g[i] * (double)t.g[i];
  s = block_sum(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}
__global__ __launch_bounds__(kThreads) void grad_norm_final_kernel(const double* part, long long count, float* norm) {
  __shared__ double red[kThreads / 64];
  double s = 0.0;
  for (long long i = threadIdx.x; i < count; i += kThreads) s += part[i];
  s = block_sum(s, red);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

long long pieces_of(int64_t n) { return (n + kPiece - 1) / kPiece; }

// Calls launch(list, pieces) for at most kPerLaunch tensors and 2^30 pieces at a time; tensors without values are left out.
template <class F>
hipError_t over_tensors(const AdamwTensor* t, int count, double lr, F&& launch) {
  AdamwList l;
  hipError_t e = hipSuccess;
  for (int k = 0; k < count && e == hipSuccess;) {
    l.count = 0;
    l.base = k;
    long long pieces = 0;
    for (; k < count && k - l.base < kPerLaunch; ++k) {
      if (pieces + pieces_of(t[k].n) > (1ll << 30) && pieces > 0) break;
      // an empty tensor keeps its place (the random bits go by it) and starts where the next one does
      l.t[l.count++] = AdamwEntry{t[k].p, t[k].g, t[k].m, t[k].v, static_cast<u8*>(t[k].e), (long long)t[k].n, (unsigned)pieces,
                                  (float)(1.0 - lr * t[k].decay)};
      pieces += pieces_of(t[k].n);
    }
    if (pieces > 0) {
      launch(l, pieces);
      e = hipGetLastError();
    }
  }
  return e;
}

}  // namespace

hipError_t launch_adamw(const AdamwTensor* t, int count, const AdamwStep& st, hipStream_t s) {
  const double c1 = 1.0 - pow(st.beta1, st.step), c2 = 1.0 - pow(st.beta2, st.step);
  const AdamwScalars c{(float)st.beta1, (float)(1.0 - st.beta1), (float)st.beta2, (float)(1.0 - st.beta2), (float)st.eps,
                       (float)(st.lr / c1), (float)(1.0 / c2), (float)st.max_norm,
                       mix_bits(mix_bits(st.seed) ^ (unsigned)st.step), st.norm};
  return over_tensors(t, count, st.lr, [&](const AdamwList& l, long long pieces) {
    if (st.bits == 8) hipLaunchKernelGGL(adamw8_kernel, dim3((unsigned)pieces), dim3(kThreads), 0, s, l, c);
    else hipLaunchKernelGGL(adamw32_kernel, dim3((unsigned)pieces), dim3(kThreads), 0, s, l, c);
  });
}

size_t grad_norm_workspace_bytes(const AdamwTensor* t, int count) {
  long long pieces = 0;
  for (int k = 0; k < count; ++k) pieces += pieces_of(t[k].n);
  return (size_t)(pieces > 0 ? pieces : 1) * sizeof(double);
}

hipError_t launch_grad_norm(const AdamwTensor* t, int count, float* norm, void* ws, hipStream_t s) {
  double* part = static_cast<double*>(ws);
  long long done = 0;
  const hipError_t e = over_tensors(t, count, 0.0, [&](const AdamwList& l, long long pieces) {
    hipLaunchKernelGGL(grad_norm_partial_kernel, dim3((unsigned)pieces), dim3(kThreads), 0, s, l, part + done);
    done += pieces;
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grad_norm_final_kernel, dim3(1), dim3(kThreads), 0, s, part, done, norm);
  return hipGetLastError();
}

hipError_t launch_adamw_state_read(const AdamwTensor* t, int count, void* const* m_out, void* const* v_out, hipStream_t s) {
  AdamwTensor o[kPerLaunch];
  for (int k = 0; k < count; k += kPerLaunch) {
    const int here = count - k < kPerLaunch ? count - k : kPerLaunch;
    for (int j = 0; j < here; ++j) {
      o[j] = t[k + j];
      o[j].p = static_cast<float*>(m_out[k + j]);
      o[j].g = static_cast<const float*>(v_out[k + j]);
    }
    const hipError_t e = over_tensors(o, here, 0.0, [&](const AdamwList& l, long long pieces) {
      hipLaunchKernelGGL(adamw_read_kernel, dim3((unsigned)pieces), dim3(kThreads), 0, s, l);
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fno
