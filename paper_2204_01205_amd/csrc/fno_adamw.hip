// One AdamW step over the tensors of a list with moments in 32 or 8 bits, the norm of their gradients, and what 8-bit
// moments stand for.
//
// All three are bound by memory: a step reads 16 and writes 12 bytes a value, with 8-bit moments 10 and 6.  The addresses of
// up to 64 tensors go with a launch's arguments, so that a list of small tensors is one launch and no table has to be kept in
// step with the gradients' addresses; a block takes 4096 values of one tensor in memory order.  354 million parameters (four
// blocks of 20 channels at 24 x 24 x 24 x 8 modes): 32 bits 1.71 ms (5.8 TB/s), 8 bits 0.97 (5.8), norm 0.21 (6.6), read of the
// 8-bit moments 0.34 (6.2); longer stretches a block 1.87 to 1.95 (32 bits), plain instead of nontemporal accesses 1.84.
//
// 8-bit moments: 256 consecutive values, four to a lane of one wave, share a power of two for each moment; a code is a small
// float relative to it.  v spans 31 powers below the largest of its block and m 15 (v is a square), both in steps of an
// eighth.  An average of decay 0.999 moves by a hundredth of such a step at a time, so that rounding to nearest would leave it
// where it is; with the bits of a float, rounding at random is one addition before the cut.
#include "fno_device.h"

#include <type_traits>

namespace fno {

namespace {

typedef unsigned char u8;
typedef unsigned short u16;
typedef unsigned v2u __attribute__((ext_vector_type(2)));

constexpr int kGroup = 256;            // values that share an exponent
constexpr int kPerLaunch = 64;         // tensors whose addresses go with one launch's arguments (3.5 KB)
constexpr int kBlockValues = 4096;     // values that a block takes at a time: 16 a thread

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
  long long piece;     // values of one tensor that a block takes: a multiple of kBlockValues
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

// Four floats, four codes or four bf16 values at an address that is 4-byte aligned.  STREAM: with the nontemporal hint, for lists
// that the memory-side cache does not hold.
template <bool STREAM>
__device__ __forceinline__ v4f load4(const float* p) {
  typedef v4f loose __attribute__((aligned(4)));
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const loose*>(p));
  else return *reinterpret_cast<const loose*>(p);
}
template <bool STREAM>
__device__ __forceinline__ void store4(float* p, v4f v) {
  typedef v4f loose __attribute__((aligned(4)));
  if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<loose*>(p));
  else *reinterpret_cast<loose*>(p) = v;
}
template <bool STREAM>
__device__ __forceinline__ void store_halves(u16* p, v2u v) {
  typedef v2u loose __attribute__((aligned(4)));
  if constexpr (STREAM) __builtin_nontemporal_store(v, reinterpret_cast<loose*>(p));
  else *reinterpret_cast<loose*>(p) = v;
}
template <bool STREAM>
__device__ __forceinline__ unsigned load_codes(const u8* p) { return ld_once<STREAM>(reinterpret_cast<const unsigned*>(p)); }
template <bool STREAM>
__device__ __forceinline__ void store_codes(u8* p, unsigned v) { st_once<STREAM>(reinterpret_cast<unsigned*>(p), v); }

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

// A thread takes 16 values at a time, four from each of four quarters of the block's, all asked for before the first is used.
template <bool STREAM>
__global__ __launch_bounds__(kThreads) void adamw32_kernel(AdamwList l, AdamwScalars c) {
  const AdamwEntry& t = l.t[tensor_of(l, blockIdx.x)];
  float scale;
  if (!clip_scale(c, scale)) return;
  const long long begin = (long long)(blockIdx.x - t.first) * l.piece;
  const long long end = begin + l.piece < t.n ? begin + l.piece : t.n;
  float *const m = static_cast<float*>(t.m), *const v = static_cast<float*>(t.v), *const p = t.p;
  const float* const g = t.g;
  long long at = begin;
  for (; at + kBlockValues <= end; at += kBlockValues) {
    v4f gq[4], mq[4], vq[4], pq[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = at + u * (kBlockValues / 4) + 4 * threadIdx.x;
      gq[u] = load4<STREAM>(g + i);
      mq[u] = load4<STREAM>(m + i);
      vq[u] = load4<STREAM>(v + i);
      pq[u] = load4<STREAM>(p + i);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = at + u * (kBlockValues / 4) + 4 * threadIdx.x;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float mi = mq[u][w], vi = vq[u][w];
        moments(c, gq[u][w] * scale, mi, vi);
        mq[u][w] = mi;
        vq[u][w] = vi;
        pq[u][w] = updated(c, t.keep, pq[u][w], mi, vi);
      }
      store4<STREAM>(m + i, mq[u]);
      store4<STREAM>(v + i, vq[u]);
      store4<STREAM>(p + i, pq[u]);
    }
  }
  for (long long i = at + threadIdx.x; i < end; i += kThreads) {
    float mi = m[i], vi = v[i];
    moments(c, g[i] * scale, mi, vi);
    m[i] = mi;
    v[i] = vi;
    p[i] = updated(c, t.keep, p[i], mi, vi);
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
// What the codes of a block have in common, the same in all lanes
struct Scale8 {
  unsigned low;        // bits of the smallest power
  unsigned first;      // bits of what m's code 1 stands for
  float part;          // that / 65536
};
__device__ __forceinline__ Scale8 scale_of(unsigned e, unsigned span) {
  Scale8 s;
  s.low = (e - span) << 3;
  s.first = (s.low + 1u) << 20;
  s.part = __builtin_bit_cast(float, s.first) * (1.0f / 65536.0f);
  return s;
}
__device__ __forceinline__ unsigned encode_m(float x, const Scale8& s, unsigned r) {
  const unsigned bits = __builtin_bit_cast(unsigned, x) & 0x7FFFFFFFu;
  const unsigned whole = min(((bits + (r << 4)) >> 20) - s.low, 127u), little = s.part * (float)r < fabsf(x) ? 1u : 0u;
  const unsigned code = bits >= s.first ? whole : little;
  return x < 0.f ? code + 128u : code;
}
__device__ __forceinline__ unsigned encode_v(float x, const Scale8& s, unsigned r) {
  const unsigned bits = __builtin_bit_cast(unsigned, x);
  const int code = (int)((bits + (r << 4)) >> 20) - (int)s.low;
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
// the largest of a wave's values, in every lane
template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_max(unsigned v) {
  return max(v, (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, ROWS == 0xF));
}
__device__ __forceinline__ unsigned wave_max(unsigned v) {
  v = dpp_max<0xB1, 0xF>(v);           // lane ^ 1
  v = dpp_max<0x4E, 0xF>(v);           // lane ^ 2
  v = dpp_max<0x141, 0xF>(v);          // mirrored in eights
  v = dpp_max<0x140, 0xF>(v);          // mirrored in rows of 16
  v = dpp_max<0x142, 0xA>(v);          // last lane of a row to the next row
  v = dpp_max<0x143, 0xC>(v);          // lane 31 to the upper half
  return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}

// One block of 256 values in a wave, four to a lane: what stays in registers between its loads and its stores.
struct Group8 {
  v4f p, g;
  unsigned m, v, e;    // codes; exponents, m's in the low byte
};
// FINE: square root and quotient to the last bit; otherwise by the instructions that are good to one unit in the last place and
// take subnormal squares for zero.
template <bool FINE>
__device__ __forceinline__ void group_step(const AdamwScalars& c, float keep, float scale, unsigned block, int lane, Group8& q) {
  const unsigned em = q.e & 255u, ev = q.e >> 8;
  float mi[4], vi[4];
  unsigned top_m = 0, top_v = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    float m = decode_m((q.m >> (8 * u)) & 255u, em), v = decode_v((q.v >> (8 * u)) & 255u, ev);
    moments(c, q.g[u] * scale, m, v);
    if (FINE) q.p[u] = updated(c, keep, q.p[u], m, v);
    else q.p[u] = q.p[u] * keep - c.lr1 * m * __builtin_amdgcn_rcpf(__builtin_amdgcn_sqrtf(v * c.ic2) + c.eps);
    top_m = max(top_m, __builtin_bit_cast(unsigned, m) & 0x7FFFFFFFu);
    top_v = max(top_v, __builtin_bit_cast(unsigned, v));
    mi[u] = m;
    vi[u] = v;
  }
  const unsigned nm = shared_exponent(wave_max(top_m), kSpanM), nv = shared_exponent(wave_max(top_v), kSpanV);
  const Scale8 sm = scale_of(nm, kSpanM), sv = scale_of(nv, kSpanV);
  q.m = 0;
  q.v = 0;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const unsigned r = mix_bits(block + (unsigned)(4 * lane + u) * 0x9E3779B1u);
    q.m |= encode_m(mi[u], sm, r & 0xFFFFu) << (8 * u);
    q.v |= encode_v(vi[u], sv, r >> 16) << (8 * u);
  }
  if (nm == 255u) q.m = 0;             // (the same in all lanes)
  if (nv == 255u) q.v = 0;
  q.e = nm | nv << 8;
}

// A wave takes four blocks of 256 values at a time, all asked for before the first is used, each stored when it is done (354 M
// values, with norm and read: 1.52 ms; all four worked side by side and stored together 1.55).
template <bool FINE, bool STREAM>
__global__ __launch_bounds__(kThreads) void adamw8_kernel(AdamwList l, AdamwScalars c) {
  const int k = tensor_of(l, blockIdx.x);
  const AdamwEntry& t = l.t[k];
  float scale;
  if (!clip_scale(c, scale)) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned key = mix_bits(c.key ^ (unsigned)(l.base + k));
  const long long begin = (long long)(blockIdx.x - t.first) * l.piece;
  const long long end = begin + l.piece < t.n ? begin + l.piece : t.n;
  u8 *const m = static_cast<u8*>(t.m), *const v = static_cast<u8*>(t.v);
  u16* const e = reinterpret_cast<u16*>(t.e);
  auto random_of = [&](long long block) { return mix_bits(mix_bits((unsigned)block + key) + (unsigned)(block >> 32)); };
  long long at = begin + wave * (kBlockValues / 4);
  for (; at + 4 * kGroup <= end; at += kBlockValues) {
    Group8 q[4];
    const long long b0 = at / kGroup;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = at + u * kGroup + 4 * lane;
      q[u].p = load4<STREAM>(t.p + i);
      q[u].g = load4<STREAM>(t.g + i);
      q[u].m = load_codes<STREAM>(m + i);
      q[u].v = load_codes<STREAM>(v + i);
      q[u].e = e[b0 + u];
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const long long i = at + u * kGroup + 4 * lane;
      group_step<FINE>(c, t.keep, scale, random_of(b0 + u), lane, q[u]);
      store4<STREAM>(t.p + i, q[u].p);
      store_codes<STREAM>(m + i, q[u].m);
      store_codes<STREAM>(v + i, q[u].v);
      if (lane == 0) e[b0 + u] = (u16)q[u].e;
    }
  }
  // the tensor's last blocks, the very last one cut: values past the end are zeros that nobody stores
  const long long stop = at + kBlockValues / 4 < end ? at + kBlockValues / 4 : end;
  for (; at < stop; at += kGroup) {
    Group8 q{};
    const long long i = at + 4 * lane;
    q.e = e[at / kGroup];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i + u >= end) continue;
      q.p[u] = t.p[i + u];
      q.g[u] = t.g[i + u];
      q.m |= (unsigned)m[i + u] << (8 * u);
      q.v |= (unsigned)v[i + u] << (8 * u);
    }
    group_step<FINE>(c, t.keep, scale, random_of(at / kGroup), lane, q);
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      if (i + u >= end) continue;
      t.p[i + u] = q.p[u];
      m[i + u] = (u8)(q.m >> (8 * u));
      v[i + u] = (u8)(q.v >> (8 * u));
    }
    if (lane == 0) e[at / kGroup] = (u16)q.e;
  }
}

// p and g of an entry hold the outputs here
template <bool STREAM>
__global__ __launch_bounds__(kThreads) void adamw_read_kernel(AdamwList l) {
  const AdamwEntry& t = l.t[tensor_of(l, blockIdx.x)];
  const long long begin = (long long)(blockIdx.x - t.first) * l.piece;
  const long long end = begin + l.piece < t.n ? begin + l.piece : t.n;
  const u8 *const m = static_cast<const u8*>(t.m), *const v = static_cast<const u8*>(t.v);
  const u16* const e = reinterpret_cast<const u16*>(t.e);
  u16 *const mo = reinterpret_cast<u16*>(t.p), *const vo = reinterpret_cast<u16*>(const_cast<float*>(t.g));
  auto put = [&](long long at, unsigned cm, unsigned cv, unsigned ex) {
    unsigned a[4], b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      a[u] = __builtin_bit_cast(unsigned, decode_m((cm >> (8 * u)) & 255u, ex & 255u));
      b[u] = __builtin_bit_cast(unsigned, decode_v((cv >> (8 * u)) & 255u, ex >> 8));
    }
    const v2u x = {a[0] >> 16 | (a[1] & 0xFFFF0000u), a[2] >> 16 | (a[3] & 0xFFFF0000u)};
    const v2u y = {b[0] >> 16 | (b[1] & 0xFFFF0000u), b[2] >> 16 | (b[3] & 0xFFFF0000u)};
    store_halves<STREAM>(mo + at, x);
    store_halves<STREAM>(vo + at, y);
  };
  long long at = begin + 4 * threadIdx.x;
  constexpr int U = kBlockValues / (4 * kThreads);
  for (; at + (U - 1) * 4 * kThreads + 4 <= end; at += kBlockValues) {
    unsigned cm[U], cv[U], ex[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      cm[u] = load_codes<STREAM>(m + at + u * 4 * kThreads);
      cv[u] = load_codes<STREAM>(v + at + u * 4 * kThreads);
      ex[u] = e[(at + u * 4 * kThreads) / kGroup];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) put(at + u * 4 * kThreads, cm[u], cv[u], ex[u]);
  }
  for (; at + 4 <= end; at += 4 * kThreads) put(at, load_codes<STREAM>(m + at), load_codes<STREAM>(v + at), e[at / kGroup]);
  for (int u = 0; u < 4; ++u) {
    if (at + u >= end) break;
    const unsigned ex = e[at / kGroup];
    mo[at + u] = (u16)(__builtin_bit_cast(unsigned, decode_m(m[at + u], ex & 255u)) >> 16);
    vo[at + u] = (u16)(__builtin_bit_cast(unsigned, decode_v(v[at + u], ex >> 8)) >> 16);
  }
}

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += red[w];
  return s;
}

// A square of a float is exact in double, and so squares of the largest and the smallest floats are neither infinite nor zero.
template <bool STREAM>
__global__ __launch_bounds__(kThreads) void grad_norm_partial_kernel(AdamwList l, double* part) {
  __shared__ double red[kThreads / 64];
  const AdamwEntry& t = l.t[tensor_of(l, blockIdx.x)];
  const long long begin = (long long)(blockIdx.x - t.first) * l.piece;
  const long long end = begin + l.piece < t.n ? begin + l.piece : t.n;
  const float* const g = t.g;
  double s[4] = {0.0, 0.0, 0.0, 0.0};
  long long at = begin;
  for (; at + kBlockValues <= end; at += kBlockValues) {
    v4f q[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) q[u] = load4<STREAM>(g + at + u * (kBlockValues / 4) + 4 * threadIdx.x);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int w = 0; w < 4; ++w) s[w] = fma((double)q[u][w], (double)q[u][w], s[w]);
  }
  for (long long i = at + threadIdx.x; i < end; i += kThreads) s[0] = fma((double)g[i], (double)g[i], s[0]);
  const double sum = block_sum((s[0] + s[1]) + (s[2] + s[3]), red);
  if (threadIdx.x == 0) part[blockIdx.x] = sum;
}
__global__ __launch_bounds__(1024) void grad_norm_final_kernel(const double* part, long long count, float* norm) {
  __shared__ double red[1024 / 64];
  double s = 0.0;
  for (long long i = threadIdx.x; i < count; i += 1024) s += part[i];
  s = block_sum(s, red);
  if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

// Whether a list with this many bytes a value is more than the memory-side cache holds.
bool streams(const AdamwTensor* t, int count, int bytes) {
  long long n = 0;
  for (int k = 0; k < count; ++k) n += t[k].n;
  return n > kStreamBytes / bytes;
}
template <class F>
void with(bool b, F&& f) {
  if (b) f(std::true_type());
  else f(std::false_type());
}

// Values that a block takes: so many that all tensors together make about `blocks` blocks, and at least kBlockValues.
long long piece_of(const AdamwTensor* t, int count, long long blocks) {
  long long n = 0;
  for (int k = 0; k < count; ++k) n += t[k].n;
  const long long rounds = (n + blocks * kBlockValues - 1) / (blocks * kBlockValues);
  return (rounds < 1 ? 1 : rounds) * kBlockValues;
}
long long pieces_of(int64_t n, long long piece) { return (n + piece - 1) / piece; }

// Calls launch(list, pieces) for at most kPerLaunch tensors and 2^23 pieces at a time.
template <class F>
hipError_t over_tensors(const AdamwTensor* t, int count, double lr, long long piece, F&& launch) {
  AdamwList l;
  hipError_t e = hipSuccess;
  for (int k = 0; k < count && e == hipSuccess;) {
    l.count = 0;
    l.base = k;
    l.piece = piece;
    long long pieces = 0;
    for (; k < count && k - l.base < kPerLaunch; ++k) {
      if (pieces + pieces_of(t[k].n, piece) > (1ll << 23) && pieces > 0) break;
      // an empty tensor keeps its place (the random bits go by it) and starts where the next one does
      l.t[l.count++] = AdamwEntry{t[k].p, t[k].g, t[k].m, t[k].v, static_cast<u8*>(t[k].e), (long long)t[k].n, (unsigned)pieces,
                                  (float)(1.0 - lr * t[k].decay)};
      pieces += pieces_of(t[k].n, piece);
    }
    if (pieces > 0) {
      launch(l, pieces);
      e = hipGetLastError();
    }
  }
  return e;
}

constexpr long long kStepBlocks = 1ll << 20;   // blocks of a step: more only where tensors are longer than 2^32 values
constexpr long long kNormBlocks = 4096;        // partial sums of the norm, and one more for every tensor

}  // namespace

hipError_t launch_adamw(const AdamwTensor* t, int count, const AdamwStep& st, hipStream_t s) {
  const double c1 = 1.0 - pow(st.beta1, st.step), c2 = 1.0 - pow(st.beta2, st.step);
  const AdamwScalars c{(float)st.beta1, (float)(1.0 - st.beta1), (float)st.beta2, (float)(1.0 - st.beta2), (float)st.eps,
                       (float)(st.lr / c1), (float)(1.0 / c2), (float)st.max_norm,
                       mix_bits(mix_bits(st.seed) ^ (unsigned)st.step), st.norm};
  return over_tensors(t, count, st.lr, piece_of(t, count, kStepBlocks), [&](const AdamwList& l, long long pieces) {
    const dim3 grid((unsigned)pieces);
    with(streams(t, count, st.bits == 8 ? 10 : 16), [&](auto stream) {
      constexpr bool S = decltype(stream)::value;
      // the root of a subnormal square is below 1.1e-19, less than half a unit in the last place of eps from 2e-12 on
      if (st.bits == 8 && st.eps >= 2e-12) hipLaunchKernelGGL((adamw8_kernel<false, S>), grid, dim3(kThreads), 0, s, l, c);
      else if (st.bits == 8) hipLaunchKernelGGL((adamw8_kernel<true, S>), grid, dim3(kThreads), 0, s, l, c);
      else hipLaunchKernelGGL(adamw32_kernel<S>, grid, dim3(kThreads), 0, s, l, c);
    });
  });
}

size_t grad_norm_workspace_bytes(const AdamwTensor* t, int count) {
  const long long piece = piece_of(t, count, kNormBlocks);
  long long pieces = 0;
  for (int k = 0; k < count; ++k) pieces += pieces_of(t[k].n, piece);
  return (size_t)(pieces > 0 ? pieces : 1) * sizeof(double);
}

hipError_t launch_grad_norm(const AdamwTensor* t, int count, float* norm, void* ws, hipStream_t s) {
  double* part = static_cast<double*>(ws);
  long long done = 0;
  const hipError_t e = over_tensors(t, count, 0.0, piece_of(t, count, kNormBlocks), [&](const AdamwList& l, long long pieces) {
    with(streams(t, count, 4), [&](auto stream) {
      hipLaunchKernelGGL(grad_norm_partial_kernel<decltype(stream)::value>, dim3((unsigned)pieces), dim3(kThreads), 0, s, l, part + done);
    });
    done += pieces;
  });
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(grad_norm_final_kernel, dim3(1), dim3(1024), 0, s, part, done, norm);
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
    const hipError_t e = over_tensors(o, here, 0.0, piece_of(o, here, kStepBlocks), [&](const AdamwList& l, long long pieces) {
      with(streams(o, here, 6), [&](auto stream) {
        hipLaunchKernelGGL(adamw_read_kernel<decltype(stream)::value>, dim3((unsigned)pieces), dim3(kThreads), 0, s, l);
      });
    });
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace fno
