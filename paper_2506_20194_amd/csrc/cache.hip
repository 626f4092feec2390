// The paged key-value cache: writing rows into it (quantised as they are written),
// reading them back, and the rotation of rows by given positions that comes
// before.
#include <hip/hip_runtime.h>

#include <cmath>

#include "cache.h"
#include "internal.h"
#include "mfma.h"

using namespace duo;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 16) == 0; }

// ---------------------------------------------------------------------------
// rotation by positions
// ---------------------------------------------------------------------------
constexpr int kMaxHalf = 128;  // pairs

// A workgroup takes `per` tokens; the cosines and sines of a token are computed once
// (the frequency theta^(-2i/head_dim) = 2^(i step), the angle in turns and its fraction in
// fp64, the rest in fp32) and shared by all of its heads through LDS.  The frequencies are
// computed here: a table of them among the arguments (1 KB) made the launch, which bounds a
// small call, 4.0 us instead of 3.5.  V: pairs per access (8 in 16-byte accesses, or 1).
// Bound: HBM; 32768 rows of 64 heads of 128 take 186 us, 5.7 TB/s read and written (a large copy
// reaches 4.95); 64 rows 5.4 us, the launch.
template <int V>
__global__ __launch_bounds__(256) void rope_at_kernel(const uint16_t* X, int64_t ldx, int64_t m, int heads, int half,
                                                      const int32_t* __restrict__ pos, double step, uint16_t* Y,
                                                      int64_t ldy, int per) {
  extern __shared__ float2 cs[];  // [token][pair]: cosine, sine
  const int64_t t0 = (int64_t)blockIdx.x * per;
  const int nt = (int)min((int64_t)per, m - t0);
  for (int e = threadIdx.x; e < nt * half; e += 256) {
    const double turn = (double)pos[t0 + e / half] * (exp2(e % half * step) * 0.15915494309189535);
    const float a = (float)((turn - rint(turn)) * 6.283185307179586);
    float sn, cn;
    sincosf(a, &sn, &cn);
    cs[e] = make_float2(cn, sn);
  }
  __syncthreads();
  const int cpr = half / V, items = nt * heads * cpr;  // accesses of half a head
  for (int e = threadIdx.x; e < items; e += 256) {
    const int c = e % cpr, h = e / cpr % heads, t = e / cpr / heads;
    const int64_t col = (int64_t)h * 2 * half + c * V;
    const uint16_t* x = X + (t0 + t) * ldx + col;
    uint16_t* y = Y + (t0 + t) * ldy + col;
    const float2* w = cs + t * half + c * V;
    if constexpr (V == 8) {
      const u32x4 a = *(const u32x4*)x, b = *(const u32x4*)(x + half);
      u32x4 ya, yb;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float a0 = __uint_as_float(a[j] << 16), a1 = __uint_as_float(a[j] & 0xffff0000u);
        const float b0 = __uint_as_float(b[j] << 16), b1 = __uint_as_float(b[j] & 0xffff0000u);
        const float2 w0 = w[2 * j], w1 = w[2 * j + 1];
        ya[j] = pack_bf16(a0 * w0.x - b0 * w0.y, a1 * w1.x - b1 * w1.y);
        yb[j] = pack_bf16(b0 * w0.x + a0 * w0.y, b1 * w1.x + a1 * w1.y);
      }
      *(u32x4*)y = ya;
      *(u32x4*)(y + half) = yb;
    } else {
      const float a = bf16_bits_to_f32(x[0]), b = bf16_bits_to_f32(x[half]);
      y[0] = f32_to_bf16_bits(a * w[0].x - b * w[0].y);
      y[half] = f32_to_bf16_bits(b * w[0].x + a * w[0].y);
    }
  }
}

// ---------------------------------------------------------------------------
// writing and reading
// ---------------------------------------------------------------------------

// Both directions: blockIdx.y is a head's K (even) or V, a thread takes 8 channels of
// kTok tokens, whose slots and rows are all loaded before the first is used.  Bound: HBM;
// a CU has some 80 vector instructions per 8 channels in the time of their bytes, which is
// why the codes are made without a division and both formats' bias rides on an addition.
// Eight heads of 128: 131072 tokens of 4 bits read in 137 us (5.0 TB/s; a token per thread
// with heads in the grid's first axis, 231) and written in 140 (4.9), of 8 bits in 162 and 165 (5.1,
// 5.0), of 16 bits 210 both ways (5.1); 16411 tokens written and read back in 8 bits in 45.
constexpr int kTok = 4;

template <int FMT, int HD>
__global__ __launch_bounds__(256) void kv_write_kernel(const uint16_t* __restrict__ K, int64_t ldk,
                                                       const uint16_t* __restrict__ V, int64_t ldv,
                                                       const int64_t* __restrict__ slots, int m, KvGeo g) {
  constexpr int C = HD / 8, T = 256 / C;  // threads per row, tokens at once
  const int which = blockIdx.y & 1, h = blockIdx.y >> 1;
  const int c = threadIdx.x % C, t0 = blockIdx.x * (T * kTok) + threadIdx.x / C;
  const uint16_t* const src = (which ? V : K) + h * HD + 8 * c;
  const int64_t ld = which ? ldv : ldk;
  int64_t slot[kTok];
  u32x4 x[kTok];
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    const int t = min(t0 + i * T, m - 1);
    slot[i] = t0 + i * T < m ? slots[t] : -1;
    x[i] = *(const u32x4*)(src + t * ld);
  }
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    const bool ok = slot[i] >= 0 && slot[i] < g.pages << g.shift;
    const KvRow<FMT, HD> row(g, ok ? slot[i] : 0, h, which);
    if constexpr (FMT == DUO_KV_BF16) {
      if (ok) *(u32x4*)(row.codes + 16 * c) = x[i];
    } else {
      uint16_t s;
      const uint2 q = kv_encode<FMT>(x[i], &s);
      if (ok) {
        if constexpr (FMT == DUO_KV_I8)
          *(uint2*)(row.codes + 8 * c) = q;
        else
          *(uint32_t*)(row.codes + 4 * c) = q.x;
        if (c % 4 == 0) *(uint16_t*)(row.scales + c / 4 * 2) = s;
      }
    }
  }
}

template <int FMT, int HD>
__global__ __launch_bounds__(256) void kv_read_kernel(KvGeo g, const int64_t* __restrict__ slots, int m,
                                                      uint16_t* __restrict__ K, int64_t ldk, uint16_t* __restrict__ V,
                                                      int64_t ldv) {
  constexpr int C = HD / 8, T = 256 / C;
  const int which = blockIdx.y & 1, h = blockIdx.y >> 1;
  const int c = threadIdx.x % C, t0 = blockIdx.x * (T * kTok) + threadIdx.x / C;
  uint16_t* const dst = (which ? V : K) + h * HD + 8 * c;
  const int64_t ld = which ? ldv : ldk;
  int64_t slot[kTok];
#pragma unroll
  for (int i = 0; i < kTok; ++i) slot[i] = slots[min(t0 + i * T, m - 1)];
  u32x4 y[kTok];
  uint2 q[kTok];
  float s[kTok];
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    const bool ok = slot[i] >= 0 && slot[i] < g.pages << g.shift;
    const KvRow<FMT, HD> row(g, ok ? slot[i] : 0, h, which);
    if constexpr (FMT == DUO_KV_BF16) {
      y[i] = *(const u32x4*)(row.codes + 16 * c);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[i][j] = ok ? y[i][j] : 0u;
    } else {
      const float v = bf16_bits_to_f32(*(const uint16_t*)(row.scales + c / 4 * 2));
      if constexpr (FMT == DUO_KV_I8)
        q[i] = *(const uint2*)(row.codes + 8 * c);
      else
        q[i].x = *(const uint32_t*)(row.codes + 4 * c);
      s[i] = ok ? v : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < kTok; ++i) {
    if (t0 + i * T >= m) break;
    if constexpr (FMT != DUO_KV_BF16) {
      constexpr float bias = KvFmt<FMT>::bias;
      float v[8];  // codes with their bias
      if constexpr (FMT == DUO_KV_I8) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)((j < 4 ? q[i].x : q[i].y) >> (8 * (j & 3)) & 255u);
      } else {
        const uint32_t even = q[i].x & 0x0f0f0f0fu, odd = q[i].x >> 4 & 0x0f0f0f0fu;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = (float)((j & 1 ? odd : even) >> (8 * (j >> 1)) & 255u);
      }
      if (__any(s[i] > 6.6e35f)) {  // a code times a scale near bf16's end may round past it
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float p = (v[j] - bias) * s[i];  // NaN stays NaN
          v[j] = fabsf(p) > 3.3895313892515355e38f ? copysignf(3.3895313892515355e38f, p) : p;
        }
      } else {  // n s - bias s is exact in fp32
        const float off = s[i] * -bias;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = fmaf(v[j], s[i], off);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) y[i][j] = pack_bf16(v[2 * j], v[2 * j + 1]);
    }
    *(u32x4*)(dst + (t0 + i * T) * ld) = y[i];
  }
}

dim3 kv_grid(int64_t m, int hd, int heads) { return dim3((unsigned)cdiv(m, 256 / (hd / 8) * kTok), 2 * heads); }

// Common checks of duo_kv_write and duo_kv_read.
duo_status rows_ok(const duo_kv_cache* c, const void* K, int64_t ldk, const void* V, int64_t ldv, const int64_t* slots,
                   int64_t m, KvGeo* g) {
  if (m < 0) return DUO_ERR_INVALID_ARG;
  if (duo_status e = kv_geo(c, g); e != DUO_OK) return e;
  const int64_t w = (int64_t)c->kv_heads * c->head_dim;
  if (ldk < w || ldv < w) return DUO_ERR_INVALID_ARG;
  if (m == 0) return DUO_OK;
  if (!K || !V || !slots) return DUO_ERR_INVALID_ARG;
  if (ldk % 8 || ldv % 8 || !aligned16(K) || !aligned16(V)) return DUO_ERR_UNSUPPORTED;
  if (m >= (int64_t)1 << 30) return DUO_ERR_UNSUPPORTED;  // fewer than 2^32 work items (kv_grid)
  return DUO_OK;
}

}  // namespace

namespace duo {

duo_status kv_geo(const duo_kv_cache* c, KvGeo* g) {
  if (!c) return DUO_ERR_INVALID_ARG;
  const size_t bytes = duo_kv_page_bytes(c->format, c->page_size, c->kv_heads, c->head_dim);
  if (bytes == 0) return c->format < 0 || c->format > DUO_KV_I4 || c->page_size < 1 || c->kv_heads < 1 || c->head_dim < 1
                             ? DUO_ERR_INVALID_ARG
                             : DUO_ERR_UNSUPPORTED;
  if (c->num_pages < 1 || !c->data) return DUO_ERR_INVALID_ARG;
  if (!aligned16(c->data)) return DUO_ERR_INVALID_ARG;
  if (c->num_pages > INT32_MAX || c->num_pages > ((int64_t)1 << 46) / (int64_t)bytes) return DUO_ERR_UNSUPPORTED;
  g->data = (uint8_t*)c->data;
  g->pages = c->num_pages;
  g->heads = c->kv_heads;
  g->block = (int64_t)(bytes / c->kv_heads);
  g->shift = 0;
  while (1 << g->shift < c->page_size) ++g->shift;
  return DUO_OK;
}

}  // namespace duo

extern "C" {

size_t duo_kv_page_bytes(int32_t format, int32_t page_size, int32_t kv_heads, int32_t head_dim) {
  if (kv_heads < 1 || kv_heads > kMaxKvHeads || (head_dim != 64 && head_dim != 128)) return 0;
  if (page_size < 16 || page_size > 256 || (page_size & (page_size - 1))) return 0;
  int row;
  switch (format) {
    case DUO_KV_BF16: row = KvFmt<DUO_KV_BF16>::row(head_dim); break;
    case DUO_KV_I8: row = KvFmt<DUO_KV_I8>::row(head_dim) + KvFmt<DUO_KV_I8>::scales(head_dim); break;
    case DUO_KV_I4: row = KvFmt<DUO_KV_I4>::row(head_dim) + KvFmt<DUO_KV_I4>::scales(head_dim); break;
    default: return 0;
  }
  return (size_t)2 * row * page_size * kv_heads;
}

duo_status duo_rope_at(const void* X, int64_t m, int64_t heads, int64_t head_dim, int64_t ldx, const int32_t* pos,
                       double theta, void* Y, int64_t ldy, void* stream) {
  if (m < 0 || heads < 1 || head_dim < 2 || (head_dim & 1) || heads > INT32_MAX || !(theta > 0.0) || !std::isfinite(theta))
    return DUO_ERR_INVALID_ARG;
  if (head_dim > 2 * kMaxHalf || heads * head_dim > INT32_MAX / 2) return DUO_ERR_UNSUPPORTED;
  if (ldx < heads * head_dim || ldy < heads * head_dim) return DUO_ERR_INVALID_ARG;
  if (m == 0) return DUO_OK;
  if (!X || !Y || !pos || (X == Y && ldx != ldy)) return DUO_ERR_INVALID_ARG;
  if (m > INT32_MAX) return DUO_ERR_UNSUPPORTED;
  const int half = (int)head_dim / 2;
  const double step = -2.0 / (double)head_dim * std::log2(theta);
  const bool vec = half % 8 == 0 && ldx % 8 == 0 && ldy % 8 == 0 && aligned16(X) && aligned16(Y);
  const int64_t items = heads * (half / (vec ? 8 : 1));  // of one token
  // an access per thread, and more where a launch would pass 2^32 work items
  const int per = (int)std::max<int64_t>({1, 256 / items, cdiv(m, kMaxGrid)});
  const dim3 grid((unsigned)cdiv(m, per));
  const size_t lds = (size_t)per * half * sizeof(float2);
  if (lds > 65536) return DUO_ERR_UNSUPPORTED;  // more rows than memory holds
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  if (vec)
    hipLaunchKernelGGL(rope_at_kernel<8>, grid, dim3(256), lds, (hipStream_t)stream, (const uint16_t*)X, ldx, m,
                       (int)heads, half, pos, step, (uint16_t*)Y, ldy, per);
  else
    hipLaunchKernelGGL(rope_at_kernel<1>, grid, dim3(256), lds, (hipStream_t)stream, (const uint16_t*)X, ldx, m,
                       (int)heads, half, pos, step, (uint16_t*)Y, ldy, per);
  DUO_LAUNCH_CHECK();
  return DUO_OK;
}

duo_status duo_kv_write(const duo_kv_cache* cache, const void* K, int64_t ldk, const void* V, int64_t ldv,
                        const int64_t* slots, int64_t m, void* stream) {
  KvGeo g;
  if (duo_status e = rows_ok(cache, K, ldk, V, ldv, slots, m, &g); e != DUO_OK) return e;
  if (m == 0) return DUO_OK;
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  return kv_by_format(cache, [&](auto fmt, auto hd) -> duo_status {
    constexpr int FMT = decltype(fmt)::value, HD = decltype(hd)::value;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_write_kernel<FMT, HD>), kv_grid(m, HD, g.heads), dim3(256), 0,
                       (hipStream_t)stream, (const uint16_t*)K, ldk, (const uint16_t*)V, ldv, slots, (int)m, g);
    DUO_LAUNCH_CHECK();
    return DUO_OK;
  });
}

duo_status duo_kv_read(const duo_kv_cache* cache, const int64_t* slots, int64_t m, void* K, int64_t ldk, void* V,
                       int64_t ldv, void* stream) {
  KvGeo g;
  if (duo_status e = rows_ok(cache, K, ldk, V, ldv, slots, m, &g); e != DUO_OK) return e;
  if (m == 0) return DUO_OK;
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  return kv_by_format(cache, [&](auto fmt, auto hd) -> duo_status {
    constexpr int FMT = decltype(fmt)::value, HD = decltype(hd)::value;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(kv_read_kernel<FMT, HD>), kv_grid(m, HD, g.heads), dim3(256), 0,
                       (hipStream_t)stream, g, slots, (int)m, (uint16_t*)K, ldk, (uint16_t*)V, ldv);
    DUO_LAUNCH_CHECK();
    return DUO_OK;
  });
}

}  // extern "C"
