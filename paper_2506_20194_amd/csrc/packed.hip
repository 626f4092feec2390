// Causal attention over packed sequences of different lengths, with grouped heads.
#include <hip/hip_runtime.h>

#include <cmath>

#include "internal.h"
#include "mfma.h"

using namespace duo;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 16) == 0; }

// One wave per row and head: lane l holds channels l and l + 64.
template <int HD>
__global__ __launch_bounds__(64) void packed_plain_kernel(const uint16_t* __restrict__ Q, int64_t ldq,
                                                          const uint16_t* __restrict__ K, int64_t ldk,
                                                          const uint16_t* __restrict__ V, int64_t ldv,
                                                          const int32_t* __restrict__ cu_q, int64_t total_q,
                                                          const int32_t* __restrict__ cu_k, int64_t total_k, int nseq,
                                                          int group, float scale, uint16_t* O, int64_t ldo) {
  const int64_t row = blockIdx.x;
  const int h = blockIdx.y, lane = threadIdx.x;
  int s = 0;
  int64_t q0 = 0, q1 = 0;
  for (; s < nseq; ++s) {
    q0 = min(max((int64_t)cu_q[s], (int64_t)0), total_q);
    q1 = min(max((int64_t)cu_q[s + 1], (int64_t)0), total_q);
    if (row >= q0 && row < q1) break;
  }
  if (s == nseq) return;
  const int64_t k0 = min(max((int64_t)cu_k[s], (int64_t)0), total_k), k1 = min(max((int64_t)cu_k[s + 1], (int64_t)0), total_k);
  const int64_t seen = min(k1 - k0, row - q0 + 1 + max(k1 - k0, (int64_t)0) - (q1 - q0));
  constexpr int E = HD / 64;
  float q[E], o[E];
  for (int e = 0; e < E; ++e) q[e] = bf16_bits_to_f32(Q[row * ldq + h * HD + lane + 64 * e]), o[e] = 0.f;
  float m = -INFINITY, l = 0.f;
  for (int64_t j = 0; j < seen; ++j) {
    float x = 0.f;
    for (int e = 0; e < E; ++e) x = fmaf(q[e], bf16_bits_to_f32(K[(k0 + j) * ldk + h / group * HD + lane + 64 * e]), x);
    for (int d = 32; d > 0; d >>= 1) x += __shfl_xor(x, d);
    x *= scale;
    const float mn = fmaxf(m, x), base = mn == -INFINITY ? 0.f : mn;
    const float f = expf(m - base), p = expf(x - base);
    m = mn;
    l = l * f + p;
    for (int e = 0; e < E; ++e) o[e] = o[e] * f + p * bf16_bits_to_f32(V[(k0 + j) * ldv + h / group * HD + lane + 64 * e]);
  }
  for (int e = 0; e < E; ++e) O[row * ldo + h * HD + lane + 64 * e] = seen > 0 ? f32_to_bf16_bits(o[e] / l) : (uint16_t)0;
}

}  // namespace

extern "C" {

duo_status duo_attention_packed(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                const int32_t* cu_q, int64_t total_q, const int32_t* cu_k, int64_t total_k,
                                int64_t nseq, int64_t heads, int64_t kv_heads, int64_t head_dim, double scale, void* O,
                                int64_t ldo, void* stream) {
  if (nseq < 0 || total_q < 0 || total_k < 0 || heads < 1 || kv_heads < 1 || head_dim < 1 || heads > 65535 ||
      kv_heads > heads || heads % kv_heads || !std::isfinite(scale))
    return DUO_ERR_INVALID_ARG;
  if (ldq < heads * head_dim || ldo < heads * head_dim || ldk < kv_heads * head_dim || ldv < kv_heads * head_dim)
    return DUO_ERR_INVALID_ARG;
  if (!cu_k && total_k != total_q) return DUO_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return DUO_ERR_UNSUPPORTED;
  if (total_q > INT32_MAX || total_k > INT32_MAX || nseq > INT32_MAX - 1) return DUO_ERR_UNSUPPORTED;
  if (nseq == 0 || total_q == 0) return DUO_OK;
  if (!Q || !O || !cu_q || (total_k > 0 && (!K || !V))) return DUO_ERR_INVALID_ARG;
  if (ldq % 8 || ldk % 8 || ldv % 8 || !aligned16(Q) || !aligned16(K) || !aligned16(V)) return DUO_ERR_UNSUPPORTED;
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  const dim3 grid((unsigned)total_q, (unsigned)heads);
  auto go = [&](auto kern) {
    hipLaunchKernelGGL(kern, grid, dim3(64), 0, (hipStream_t)stream, (const uint16_t*)Q, ldq, (const uint16_t*)K, ldk,
                       (const uint16_t*)V, ldv, cu_q, total_q, cu_k ? cu_k : cu_q, total_k, (int)nseq,
                       (int)(heads / kv_heads), (float)scale, (uint16_t*)O, ldo);
  };
  head_dim == 128 ? go(packed_plain_kernel<128>) : go(packed_plain_kernel<64>);
  DUO_LAUNCH_CHECK();
  return DUO_OK;
}

}  // extern "C"
