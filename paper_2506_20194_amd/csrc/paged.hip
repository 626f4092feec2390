// Attention of one query per sequence over the paged key-value cache.
#include <hip/hip_runtime.h>

#include <cmath>

#include "cache.h"
#include "internal.h"
#include "mfma.h"

using namespace duo;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 16) == 0; }

template <int FMT, int HD>
__device__ float kv_number(const uint8_t* blk, int which, int shift, int row, int ch) {
  const uint8_t* p = blk + kv_rows_at<FMT, HD>(which, shift) + row * KvFmt<FMT>::row(HD);
  if constexpr (FMT == DUO_KV_BF16) {
    return bf16_bits_to_f32(*(const uint16_t*)(p + 2 * ch));
  } else {
    const float s = bf16_bits_to_f32(*(const uint16_t*)(blk + kv_scales_at<FMT, HD>(which, shift) +
                                                        row * KvFmt<FMT>::scales(HD) + ch / kKvGroup * 2));
    const int n = FMT == DUO_KV_I8 ? p[ch] : p[ch / 2] >> (4 * (ch & 1)) & 15;
    return (float)(n - KvFmt<FMT>::bias) * s;
  }
}

// One wave per sequence and head: lane l holds channels l and l + 64.
template <int FMT, int HD>
__global__ __launch_bounds__(64) void paged_plain_kernel(const uint16_t* __restrict__ Q, int64_t ldq, KvGeo g,
                                                         const int32_t* __restrict__ table, int64_t ldt,
                                                         const int32_t* __restrict__ lens, int max_len, int group,
                                                         float scale, uint16_t* O, int64_t ldo) {
  const int64_t s = blockIdx.x;
  const int h = blockIdx.y, lane = threadIdx.x;
  const int len = min(max(lens[s], 0), max_len);
  constexpr int E = HD / 64;
  float q[E], o[E];
  for (int e = 0; e < E; ++e) q[e] = bf16_bits_to_f32(Q[s * ldq + h * HD + lane + 64 * e]), o[e] = 0.f;
  float m = -INFINITY, l = 0.f;
  for (int j = 0; j < len; ++j) {
    const int page = table[s * ldt + (j >> g.shift)];
    if (page < 0 || page >= g.pages) {
      l = NAN;
      break;
    }
    const uint8_t* blk = g.data + ((int64_t)page * g.heads + h / group) * g.block;
    const int row = j & ((1 << g.shift) - 1);
    float x = 0.f;
    for (int e = 0; e < E; ++e) x = fmaf(q[e], kv_number<FMT, HD>(blk, 0, g.shift, row, lane + 64 * e), x);
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    x *= scale;
    const float mn = fmaxf(m, x), base = mn == -INFINITY ? 0.f : mn;
    const float f = expf(m - base), p = expf(x - base);
    m = mn;
    l = l * f + p;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + p * kv_number<FMT, HD>(blk, 1, g.shift, row, lane + 64 * e);
  }
  for (int e = 0; e < E; ++e) O[s * ldo + h * HD + lane + 64 * e] = len > 0 ? f32_to_bf16_bits(o[e] / l) : (uint16_t)0;
}

}  // namespace

extern "C" {

size_t duo_attention_paged_workspace_size(int64_t nseq, int64_t heads, int64_t kv_heads, int64_t head_dim,
                                          int64_t max_len) {
  return 0;
}

duo_status duo_attention_paged(const void* Q, int64_t ldq, const duo_kv_cache* cache, const int32_t* table, int64_t ldt,
                               const int32_t* lens, int64_t nseq, int64_t max_len, int64_t heads, double scale, void* O,
                               int64_t ldo, void* ws, size_t ws_bytes, void* stream) {
  KvGeo g;
  if (duo_status e = kv_geo(cache, &g); e != DUO_OK) return e;
  const int hd = cache->head_dim;
  if (nseq < 0 || max_len < 0 || heads < 1 || heads > 65535 || heads % g.heads || !std::isfinite(scale) ||
      ldq < heads * hd || ldo < heads * hd || ldt < 0 || ldt < cdiv(max_len, cache->page_size))
    return DUO_ERR_INVALID_ARG;
  if (nseq > INT32_MAX || max_len > INT32_MAX - 1024) return DUO_ERR_UNSUPPORTED;
  if (nseq == 0) return DUO_OK;
  if (!Q || !O || !lens || (max_len > 0 && !table)) return DUO_ERR_INVALID_ARG;
  if (ldq % 8 || !aligned16(Q)) return DUO_ERR_UNSUPPORTED;
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  return kv_by_format(cache, [&](auto fmt, auto dim) -> duo_status {
    constexpr int FMT = decltype(fmt)::value, HD = decltype(dim)::value;
    hipLaunchKernelGGL(HIP_KERNEL_NAME(paged_plain_kernel<FMT, HD>), dim3((unsigned)nseq, (unsigned)heads), dim3(64), 0,
                       (hipStream_t)stream, (const uint16_t*)Q, ldq, g, table, ldt, lens, (int)max_len,
                       (int)(heads / g.heads), (float)scale, (uint16_t*)O, ldo);
    DUO_LAUNCH_CHECK();
    return DUO_OK;
  });
}

}  // extern "C"
