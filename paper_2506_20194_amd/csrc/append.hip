// Head norms with the rotation by positions in one pass over the rows, and the same
// for a step's keys on their way into the paged cache, with its queries beside them.
//
// A head x of head_dim numbers at position p becomes
//   y = x / sqrt(mean(x^2) + eps) * gain    (where it has a norm)
//   z_i = y_i cos(p f_i) - y_{i+half} sin(p f_i),  z_{i+half} = y_{i+half} cos(p f_i) + y_i sin(p f_i)
// with f_i = theta^(-2i / head_dim), in fp32 but for the angle (fp64), rounded to bf16 once.  What
// goes into an 8- or 4-bit cache are the codes of that bf16 row: an appended key is, bit
// for bit, the one that rotating and writing it by two calls would have stored, and kv_encode's
// argument needs numbers of eight bits.  (Codes of the fp32 row would have an error
// lower by 4 % in 8 bits and 0.02 % in 4, on normally distributed numbers.)
//
// A thread takes eight pairs (16 bytes of each half of a head), a head's threads are
// neighbours, which add up its squares by shuffles; the angles of a token are computed once
// for all of its heads and shared through LDS.
//
// Bound: HBM, every row read and written once (a large copy reaches 6.0 TB/s).  Norms and rotation
// of 16384 tokens of 64 heads of 128 95 us, 5.7 TB/s; few tokens 6.5 us with the call from Python.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cache.h"
#include "internal.h"
#include "mfma.h"

using namespace duo;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 16) == 0; }

constexpr int kMaxHalf = 128;  // pairs

// Cosines and sines of nt tokens' angles, as rope_at_kernel has them.
__device__ __forceinline__ void angles(float2* cs, const int32_t* __restrict__ pos, int64_t t0, int nt, int half, double step) {
  for (int e = threadIdx.x; e < nt * half; e += 256) {
    const double turn = (double)pos[t0 + e / half] * (exp2(e % half * step) * 0.15915494309189535);
    const float a = (float)((turn - rint(turn)) * 6.283185307179586);
    float sn, cn;
    sincosf(a, &sn, &cn);
    cs[e] = make_float2(cn, sn);
  }
}

__device__ __forceinline__ void load_gain(float* to, const void* gain, int f32, int n) {
  for (int e = threadIdx.x; e < n; e += 256)
    to[e] = !gain ? 1.f : f32 ? ((const float*)gain)[e] : bf16_bits_to_f32(((const uint16_t*)gain)[e]);
}

// Eight pairs: a the first of each, b the second.
struct Pairs {
  float a[8], b[8];
  __device__ __forceinline__ Pairs(const u32x4& x, const u32x4& y) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      a[2 * j] = __uint_as_float(x[j] << 16), a[2 * j + 1] = __uint_as_float(x[j] & 0xffff0000u);
      b[2 * j] = __uint_as_float(y[j] << 16), b[2 * j + 1] = __uint_as_float(y[j] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ float squares() const {
    float s = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) s = fmaf(a[j], a[j], fmaf(b[j], b[j], s));
    return s;
  }
  // times r and the gains of both halves
  __device__ __forceinline__ void scale(float r, const float* ga, const float* gb) {
#pragma unroll
    for (int j = 0; j < 8; ++j) a[j] = a[j] * r * ga[j], b[j] = b[j] * r * gb[j];
  }
  __device__ __forceinline__ void turn(const float2* w, u32x4* x, u32x4* y) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 w0 = w[2 * j], w1 = w[2 * j + 1];
      (*x)[j] = pack_bf16(a[2 * j] * w0.x - b[2 * j] * w0.y, a[2 * j + 1] * w1.x - b[2 * j + 1] * w1.y);
      (*y)[j] = pack_bf16(b[2 * j] * w0.x + a[2 * j] * w0.y, b[2 * j + 1] * w1.x + a[2 * j + 1] * w1.y);
    }
  }
};

// ---------------------------------------------------------------------------
// rows to rows
// ---------------------------------------------------------------------------
struct NormArgs {
  const uint16_t* X;
  uint16_t* Y;
  int64_t ldx, ldy, m;
  const int32_t* pos;
  const void* gain;
  double step;
  float eps;
  int gain_f32, heads, half, per;
  int lanes;  // of a head: half / 8 rounded up to a power of two
};

// A workgroup takes `per` tokens.  Heads whose half is no power of two leave some of their
// lanes idle.
__global__ __launch_bounds__(256) void norm_rope_kernel(NormArgs g) {
  extern __shared__ float2 cs[];  // [token][pair], then the gains
  float* const gain = (float*)(cs + g.per * g.half);
  const int64_t t0 = (int64_t)blockIdx.x * g.per;
  const int nt = (int)min((int64_t)g.per, g.m - t0);
  load_gain(gain, g.gain, g.gain_f32, 2 * g.half);
  angles(cs, g.pos, t0, nt, g.half, g.step);
  __syncthreads();
  const int items = nt * g.heads * g.lanes;
  for (int e = threadIdx.x; e < items; e += 256) {
    const int c = e & (g.lanes - 1), r = e / g.lanes, h = r % g.heads, t = r / g.heads;
    const bool live = 8 * c < g.half;
    const int64_t col = (int64_t)h * 2 * g.half + (live ? 8 * c : 0);
    const uint16_t* const x = g.X + (t0 + t) * g.ldx + col;
    Pairs p(*(const u32x4*)x, *(const u32x4*)(x + g.half));
    float s = live ? p.squares() : 0.f;
    for (int o = 1; o < g.lanes; o <<= 1) s += __shfl_xor(s, o);
    if (!live) continue;
    p.scale(rsqrtf(s / (float)(2 * g.half) + g.eps), gain + 8 * c, gain + g.half + 8 * c);
    u32x4 a, b;
    p.turn(cs + t * g.half + 8 * c, &a, &b);
    uint16_t* const y = g.Y + (t0 + t) * g.ldy + col;
    *(u32x4*)y = a;
    *(u32x4*)(y + g.half) = b;
  }
}

// The same for any even head_dim, stride and alignment: a workgroup per token, a wave per head, numbers of 2 bytes one
// by one, as rows may begin anywhere.  16384 tokens of 64 heads of 100 265 us (1.6 TB/s), of 128 in rows that begin 2 bytes
// behind a multiple of 16 282 us, 104 where they do not; heads whose half is no multiple of 8 channels are rare.
__global__ __launch_bounds__(256) void norm_rope_plain_kernel(NormArgs g) {
  extern __shared__ float2 cs[];
  float* const gain = (float*)(cs + g.half);
  const int lane = threadIdx.x & 63;
  for (int64_t t = blockIdx.x; t < g.m; t += gridDim.x) {
    __syncthreads();
    load_gain(gain, g.gain, g.gain_f32, 2 * g.half);
    angles(cs, g.pos, t, 1, g.half, g.step);
    __syncthreads();
    for (int h = threadIdx.x >> 6; h < g.heads; h += 4) {
      const uint16_t* const x = g.X + t * g.ldx + (int64_t)h * 2 * g.half;
      uint16_t* const y = g.Y + t * g.ldy + (int64_t)h * 2 * g.half;
      float a[kMaxHalf / 64], b[kMaxHalf / 64], s = 0.f;
#pragma unroll
      for (int i = 0; i < kMaxHalf / 64; ++i) {
        const int c = 64 * i + lane;
        a[i] = c < g.half ? bf16_bits_to_f32(x[c]) : 0.f;
        b[i] = c < g.half ? bf16_bits_to_f32(x[c + g.half]) : 0.f;
        s = fmaf(a[i], a[i], fmaf(b[i], b[i], s));
      }
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) s += __shfl_xor(s, o);
      const float r = rsqrtf(s / (float)(2 * g.half) + g.eps);
#pragma unroll
      for (int i = 0; i < kMaxHalf / 64; ++i) {
        const int c = 64 * i + lane;
        if (c >= g.half) break;
        const float u = a[i] * r * gain[c], v = b[i] * r * gain[c + g.half];
        y[c] = f32_to_bf16_bits(u * cs[c].x - v * cs[c].y);
        y[c + g.half] = f32_to_bf16_bits(v * cs[c].x + u * cs[c].y);
      }
    }
  }
}

// ---------------------------------------------------------------------------
// rows into the cache
// ---------------------------------------------------------------------------
struct AppendArgs {
  const uint16_t *K, *V, *Q;
  uint16_t* Y;
  int64_t ldk, ldv, ldq, ldy, m;
  const int64_t* slots;
  const int32_t* pos;
  const void *k_gain, *q_gain;
  KvGeo kv;
  double step;
  float eps;  // < 0: no norms
  int gain_f32, heads, per;
};

// A token's heads one behind the other: those of Q, of K, of V.  One launch instead of one for Q, one for
// K and a write: 32 tokens, 64 heads on 8 of 128, 11.6 us and 23.2 (calls from Python), 16411 into 8 bits 125 and 136
// (5.1 TB/s; the rows' codes cost vector instructions beside the rotation), into 16 bits 124 and 140.
template <int FMT, int HD>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs g) {
  constexpr int HALF = HD / 2, C = HALF / 8;
  extern __shared__ float2 cs[];  // [token][pair]
  __shared__ float gain[2][HD];   // of Q, of K
  const int64_t t0 = (int64_t)blockIdx.x * g.per;
  const int nt = (int)min((int64_t)g.per, g.m - t0);
  const bool norm = g.eps >= 0.f;
  const int hs = g.heads + 2 * g.kv.heads, items = nt * hs * C;
  if (norm) {
    load_gain(gain[0], g.q_gain, g.gain_f32, g.heads ? HD : 0);
    load_gain(gain[1], g.k_gain, g.gain_f32, HD);
  }
  angles(cs, g.pos, t0, nt, HALF, g.step);
  __syncthreads();
  for (int e = threadIdx.x; e < items; e += 256) {
    const int c = e % C, r = e / C, h = r % hs, t = r / hs;
    // 0: a head of Q, 1: of K, 2: of V
    const int kind = h < g.heads ? 0 : h < g.heads + g.kv.heads ? 1 : 2;
    const int hh = kind == 0 ? h : h - g.heads - (kind - 1) * g.kv.heads;
    const int col = hh * HD + 8 * c;
    const uint16_t* const x = kind == 0 ? g.Q + (t0 + t) * g.ldq + col : kind == 1 ? g.K + (t0 + t) * g.ldk + col : g.V + (t0 + t) * g.ldv + col;
    u32x4 a = *(const u32x4*)x, b = *(const u32x4*)(x + HALF);
    if (kind < 2) {
      Pairs p(a, b);
      if (norm) {
        float s = p.squares();
#pragma unroll
        for (int o = 1; o < C; o <<= 1) s += __shfl_xor(s, o);
        p.scale(rsqrtf(s / (float)HD + g.eps), gain[kind] + 8 * c, gain[kind] + HALF + 8 * c);
      }
      p.turn(cs + t * HALF + 8 * c, &a, &b);
    }
    if (kind == 0) {
      uint16_t* const y = g.Y + (t0 + t) * g.ldy + col;
      *(u32x4*)y = a;
      *(u32x4*)(y + HALF) = b;
      continue;
    }
    const int64_t slot = g.slots[t0 + t];
    const bool ok = slot >= 0 && slot < g.kv.pages << g.kv.shift;
    const KvRow<FMT, HD> row(g.kv, ok ? slot : 0, hh, kind - 1);
    if constexpr (FMT == DUO_KV_BF16) {
      if (ok) {
        *(u32x4*)(row.codes + 16 * c) = a;
        *(u32x4*)(row.codes + 16 * (c + C)) = b;
      }
    } else {
      // four threads in a row hold the 32 channels of a group, in either half
      uint16_t sa, sb;
      const uint2 qa = kv_encode<FMT>(a, &sa), qb = kv_encode<FMT>(b, &sb);
      if (ok) {
        if constexpr (FMT == DUO_KV_I8) {
          *(uint2*)(row.codes + 8 * c) = qa;
          *(uint2*)(row.codes + 8 * (c + C)) = qb;
        } else {
          *(uint32_t*)(row.codes + 4 * c) = qa.x;
          *(uint32_t*)(row.codes + 4 * (c + C)) = qb.x;
        }
        if (c % 4 == 0) {
          *(uint16_t*)(row.scales + c / 4 * 2) = sa;
          *(uint16_t*)(row.scales + (c + C) / 4 * 2) = sb;
        }
      }
    }
  }
}

bool theta_ok(double theta) { return theta > 0.0 && std::isfinite(theta); }
bool gain_type_ok(int32_t t) { return t == DUO_F32 || t == DUO_BF16; }

// Tokens of a workgroup.
int tokens_of(int64_t m, int64_t items) {
  return (int)std::max<int64_t>({1, 256 / items, cdiv(m, kMaxGrid)});
}

}  // namespace

extern "C" {

duo_status duo_head_norm_rope(const void* X, int64_t m, int64_t heads, int64_t head_dim, int64_t ldx, const int32_t* pos,
                              const void* gain, int32_t gain_dtype, double eps, double theta, void* Y, int64_t ldy,
                              void* stream) {
  if (m < 0 || heads < 1 || head_dim < 2 || (head_dim & 1) || heads > INT32_MAX || !theta_ok(theta) || !(eps >= 0.0) ||
      !std::isfinite(eps) || (gain && !gain_type_ok(gain_dtype)))
    return DUO_ERR_INVALID_ARG;
  if (head_dim > 2 * kMaxHalf || heads * head_dim > INT32_MAX / 4) return DUO_ERR_UNSUPPORTED;
  if (ldx < heads * head_dim || ldy < heads * head_dim) return DUO_ERR_INVALID_ARG;
  if (m == 0) return DUO_OK;
  if (!X || !Y || !pos || (X == Y && ldx != ldy)) return DUO_ERR_INVALID_ARG;
  if (m > INT32_MAX) return DUO_ERR_UNSUPPORTED;
  NormArgs g = {};
  g.X = (const uint16_t*)X, g.Y = (uint16_t*)Y;
  g.ldx = ldx, g.ldy = ldy, g.m = m;
  g.pos = pos, g.gain = gain, g.gain_f32 = gain_dtype == DUO_F32;
  g.step = -2.0 / (double)head_dim * std::log2(theta);
  g.eps = (float)eps, g.heads = (int)heads, g.half = (int)head_dim / 2;
  const hipStream_t s = (hipStream_t)stream;
  if (g.half % 8 == 0 && ldx % 8 == 0 && ldy % 8 == 0 && aligned16(X) && aligned16(Y)) {
    g.lanes = 1;
    while (8 * g.lanes < g.half) g.lanes *= 2;
    g.per = tokens_of(m, heads * g.lanes);
    const size_t lds = ((size_t)g.per + 1) * g.half * sizeof(float2);
    if (lds > 65536) return DUO_ERR_UNSUPPORTED;  // more rows than memory holds
    if (duo_status d = device_ok(); d != DUO_OK) return d;
    hipLaunchKernelGGL(norm_rope_kernel, dim3((unsigned)cdiv(m, g.per)), dim3(256), lds, s, g);
  } else {
    if (duo_status d = device_ok(); d != DUO_OK) return d;
    hipLaunchKernelGGL(norm_rope_plain_kernel, dim3((unsigned)std::min(m, kMaxGrid)), dim3(256),
                       2 * g.half * sizeof(float2), s, g);
  }
  DUO_LAUNCH_CHECK();
  return DUO_OK;
}

duo_status duo_kv_append(const duo_kv_cache* cache, const void* K, int64_t ldk, const void* V, int64_t ldv,
                         const int64_t* slots, const int32_t* pos, int64_t m, double theta, double eps, const void* k_gain,
                         const void* Q, int64_t ldq, int64_t heads, const void* q_gain, int32_t gain_dtype, void* Y,
                         int64_t ldy, void* stream) {
  if (m < 0 || heads < 0 || heads > 65535 || !theta_ok(theta) || !std::isfinite(eps) ||
      ((k_gain || q_gain) && (!gain_type_ok(gain_dtype) || eps < 0.0)) || (q_gain && heads == 0))
    return DUO_ERR_INVALID_ARG;
  AppendArgs g = {};
  if (duo_status e = kv_geo(cache, &g.kv); e != DUO_OK) return e;
  const int64_t hd = cache->head_dim, w = g.kv.heads * hd;
  if (ldk < w || ldv < w || (heads > 0 && (ldq < heads * hd || ldy < heads * hd))) return DUO_ERR_INVALID_ARG;
  if (m == 0) return DUO_OK;
  if (!K || !V || !slots || !pos || (heads > 0 && (!Q || !Y || (Q == Y && ldq != ldy)))) return DUO_ERR_INVALID_ARG;
  if (ldk % 8 || ldv % 8 || !aligned16(K) || !aligned16(V)) return DUO_ERR_UNSUPPORTED;
  if (heads > 0 && (ldq % 8 || ldy % 8 || !aligned16(Q) || !aligned16(Y))) return DUO_ERR_UNSUPPORTED;
  if (m > INT32_MAX) return DUO_ERR_UNSUPPORTED;
  g.K = (const uint16_t*)K, g.V = (const uint16_t*)V, g.Q = (const uint16_t*)Q, g.Y = (uint16_t*)Y;
  g.ldk = ldk, g.ldv = ldv, g.ldq = ldq, g.ldy = ldy, g.m = m;
  g.slots = slots, g.pos = pos, g.k_gain = k_gain, g.q_gain = q_gain;
  g.step = -2.0 / (double)hd * std::log2(theta);
  g.eps = eps < 0.0 ? -1.f : (float)eps;
  g.gain_f32 = gain_dtype == DUO_F32, g.heads = (int)heads;
  g.per = tokens_of(m, (heads + 2 * g.kv.heads) * (hd / 16));
  const size_t lds = (size_t)g.per * (hd / 2) * sizeof(float2);
  if (lds > 61440) return DUO_ERR_UNSUPPORTED;  // more rows than memory holds
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  return kv_by_format(cache, [&](auto fmt, auto dim) -> duo_status {
    constexpr int FMT = decltype(fmt)::value, HD = decltype(dim)::value;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(append_kernel<FMT, HD>), dim3((unsigned)cdiv(m, g.per)), dim3(256), lds,
                       (hipStream_t)stream, g);
    DUO_LAUNCH_CHECK();
    return DUO_OK;
  });
}

}  // extern "C"
