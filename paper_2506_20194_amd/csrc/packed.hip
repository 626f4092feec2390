// Causal attention over packed sequences of different lengths, with grouped heads, in
// one pass over the keys with a running maximum and sum.
//
// One workgroup per (sequence, query head, block of 32 NW queries); wave w owns queries
// 32 w .. 32 w + 31.  Everything is computed transposed, with v_mfma_f32_32x32x16_bf16
// (lane l holds row l % 32 of A and column l % 32 of B, the 8 consecutive k of half
// l / 32; accumulator element r sits at row 8 (r / 4) + 4 (l / 32) + r % 4, column
// l % 32):
//   S^T = K Q^T    a lane's 16 elements per block of 32 keys belong to one query;
//   O^T = V^T P^T  P^T's fragments are the lane's own probabilities, V^T's take the
//                  same keys from the row-major V tile with transposing LDS reads.
// K and V tiles of 64 keys stream global -> LDS directly, two buffers each.
//
// Probabilities are taken relative to a running reference that is moved (and O and the
// sum with it) only when a score exceeds it by more than 8 in the exponent of two:
// they then stay below 2^8, which costs no accuracy in fp32 or bf16.
//
// Unseen keys get probability 0, and 0 times a value that is not finite would not be
// 0: tiles in which some query does not see some key are searched for such values,
// and where there are any they enter as zeros, and what is seen of them is counted with
// two more products (see poison).
#include <hip/hip_runtime.h>

#include <cmath>

#include "internal.h"
#include "mfma.h"
#include "pingpong.h"

using namespace duo;
using namespace duo::pp;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 16) == 0; }

struct PackedArgs {
  const uint16_t *Q, *K, *V;
  uint16_t* O;
  int64_t ldq, ldk, ldv, ldo;
  const int32_t *cu_q, *cu_k;
  int total_q, total_k, nseq, kv_heads, group;
  int blocks;  // bound of the blocks of queries of one head
  float cexp;  // exp(s scale) = 2^(s cexp), with the queries' signs turned for a negative scale
  uint32_t flip;
  int vec;  // 8-byte stores of O
};

__device__ inline int cut(int v, int total) { return min(max(v, 0), total); }

// Of workgroup `id`: its query head, and which block of queries counted through all
// sequences.  Ids go round-robin over the XCDs: a K/V head lives on 8 / e of them, e =
// gcd(kv_heads, 8), which take its blocks in turn, all heads of a group one after the
// other, so that they share K and V in that L2.
__device__ inline bool place(int id, const PackedArgs& a, int* head, int* block) {
  const int x = id & 7, e = a.kv_heads & -a.kv_heads & 7 ? a.kv_heads & -a.kv_heads & 7 : 8, sh = 8 / e;
  int j = id >> 3;
  const int g = j % a.group;
  j /= a.group;
  const int per = (a.blocks + sh - 1) / sh;  // blocks of one K/V head here
  const int kv = j / per * e + x % e;
  *head = kv * a.group + g;
  *block = j % per * sh + x / e;
  return kv < a.kv_heads && *block < a.blocks;
}

// The sequence and the block within it (the last block first) of block b; false past the last.
template <int QB>
__device__ inline bool find(const PackedArgs& a, int b, int* seq, int* qb) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < a.nseq; s0 += 64) {
    const int s = s0 + lane;
    int n = 0;
    if (s < a.nseq) n = (max(cut(a.cu_q[s + 1], a.total_q) - cut(a.cu_q[s], a.total_q), 0) + QB - 1) / QB;
    int up = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(up, o);
      if (lane >= o) up += v;
    }
    const uint64_t past = __ballot(up > b);
    if (past) {
      const int l = __ffsll((unsigned long long)past) - 1;
      *seq = s0 + l;
      *qb = __builtin_amdgcn_readlane(up, l) - 1 - b;
      return true;
    }
    b -= __builtin_amdgcn_readlane(up, 63);
    if (b < 0) return false;
  }
  return false;
}

template <int HD, int NW>
__global__ __launch_bounds__(64 * NW, NW / 2) void packed_kernel(PackedArgs a) {
  constexpr int KB = 64;                // keys per tile
  constexpr int CH = HD / 8;            // 16-byte chunks per key row
  constexpr int KS = HD / 16;           // MFMA steps over head_dim
  constexpr int DB = HD / 32;           // 32-wide blocks of the output row
  constexpr int TILE = KB * CH;         // chunks per operand tile
  constexpr int NL = TILE / (64 * NW);  // 16-byte loads per thread, operand and tile
  constexpr int QB = 32 * NW;
  __shared__ u32x4 sm[2][2][TILE];      // [buffer][K, V]
  int head, block, s, qb;
  if (!place(blockIdx.x, a, &head, &block) || !find<QB>(a, block, &s, &qb)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int l32 = lane & 31, half = lane >> 5;
  const int q_first = cut(a.cu_q[s], a.total_q), lq = cut(a.cu_q[s + 1], a.total_q) - q_first;
  const int k_first = cut(a.cu_k[s], a.total_k), lk = max(cut(a.cu_k[s + 1], a.total_k) - k_first, 0);
  const int off = lk - lq;              // query i sees keys j <= i + off
  const int q0 = qb * QB, qw = q0 + 32 * wave;
  const uint16_t* const Kh = a.K + (int64_t)k_first * a.ldk + head / a.group * HD;
  const uint16_t* const Vh = a.V + (int64_t)k_first * a.ldv + head / a.group * HD;
  // chunk c of key row r sits at position kswz(r, c) (vswz) of its row: 16 consecutive
  // keys' chunks of a K fragment, and the four keys x 64 bytes that half a wave's
  // transposing read of V touches, cover the 64 banks once
  auto kswz = [](int key, int c) { return CH == 16 ? c ^ (key & 15) : c ^ ((key >> 1) & 7); };
  auto vswz = [](int key, int c) { return CH == 16 ? c ^ (4 * (key & 3)) : c ^ (4 * ((key >> 1) & 1)); };

  u32x4 qa[KS];
  {
    const uint16_t* q = a.Q + (int64_t)(q_first + min(qw + l32, lq - 1)) * a.ldq + head * HD;
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      qa[c] = *(const u32x4*)(q + 8 * (2 * c + half));
#pragma unroll
      for (int j = 0; j < 4; ++j) qa[c][j] ^= a.flip;
    }
  }
  const int seen = min(q0 + QB, lq) + off;  // keys that the block's last query sees
  const int nkb = (seen + KB - 1) / KB;     // <= 0: none
  auto issue = [&](const uint16_t* src, int64_t ld, int kb, u32x4* dst, bool is_v) {
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int base = (wave * NL + i) * 64;  // wave-uniform destination
      const int key = (base + lane) / CH, p = (base + lane) % CH;
      const int64_t at = (int64_t)min(kb * KB + key, lk - 1) * ld;
      __builtin_amdgcn_global_load_lds((const void*)(src + at + 8 * (is_v ? vswz(key, p) : kswz(key, p))),
                                       (__attribute__((address_space(3))) void*)(dst + base), 16, 0, 0);
    }
  };

  float m = -INFINITY, mc = -INFINITY, l = 0.f;  // reference, times cexp; sum of this half's keys
  f16x o[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  // transposing read: lane i of each 16 addresses key i / 4, 4 values at 4 (i % 4)
  const int tj = (lane & 15) >> 2;
  int vo[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d)
    vo[d] = (4 * half + tj) * HD * 2 + vswz(tj, 4 * d + 2 * ((lane >> 4) & 1)) * 16 + (lane & 3) * 8;
  typedef __attribute__((address_space(3))) s16v4 lds4;
  auto read_v = [&](const uint8_t* sV, int t, int d) {
    const s16v4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(sV + vo[d] + (16 * t) * HD * 2));
    const s16v4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(sV + vo[d] + (16 * t + 8) * HD * 2));
    u32x4 v;
    __builtin_memcpy(&v, &v0, 8);
    __builtin_memcpy((char*)&v + 8, &v1, 8);
    return v;
  };
  auto key_of = [&](int b, int r) { return 32 * b + 8 * (r >> 2) + 4 * half + (r & 3); };

  if (nkb > 0) {
    issue(Kh, a.ldk, 0, sm[0][0], false);
    issue(Vh, a.ldv, 0, sm[0][1], true);
  }
  for (int kb = 0; kb < nkb; ++kb) {
    wait_vm<0>();   // this wave's part of the tiles landed
    lds_barrier();  // every wave's; and every wave is done with the tiles before
    if (kb + 1 < nkb) {
      issue(Kh, a.ldk, kb + 1, sm[(kb + 1) & 1][0], false);
      issue(Vh, a.ldv, kb + 1, sm[(kb + 1) & 1][1], true);
    }
    if (kb * KB > qw + 31 + off) continue;  // uniform per wave: every key lies above its queries
    const u32x4* sK = sm[kb & 1][0];
    const uint8_t* sV = (const uint8_t*)sm[kb & 1][1];
    f16x sc[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[b][r] = 0.f;
      const int key = 32 * b + l32;
#pragma unroll
      for (int c = 0; c < KS; ++c) sc[b] = mma32_bf16(sK[key * CH + kswz(key, 2 * c + half)], qa[c], sc[b]);
    }
    const bool masked = kb * KB + KB - 1 > qw + off;  // uniform per wave: some query does not see some key
    const int see = qw + l32 + off - kb * KB;         // this lane's query sees keys 0 .. see of the tile
    if (masked) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key_of(b, r) > see) sc[b][r] = -INFINITY;
    }
    float mt = sc[0][0];
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) mt = fmaxf(mt, sc[b][r]);
    {
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
      mt = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    }
    // a new reference where the scores leave the old one's range
    if (__any(mt > m && !(mt * a.cexp <= mc + 8.f))) {
      const bool up = mt > m && !(mt * a.cexp <= mc + 8.f);
      const float mcn = up ? mt * a.cexp : mc;
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - mcn);
      m = up ? mt : m;
      mc = mcn;
      l = m == -INFINITY ? l : l * f;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= f;
    }
    const float base = m == -INFINITY ? 0.f : mc;
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[b][r] = __builtin_amdgcn_exp2f(fmaf(sc[b][r], a.cexp, -base));
    bool poison = false;
    if (masked) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (key_of(b, r) > see) sc[b][r] = 0.f;
      uint32_t any = 0;
#pragma unroll
      for (int i = 0; i < TILE / 64; ++i) {
        const u32x4 v = ((const u32x4*)sV)[i * 64 + lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) any |= ((v[j] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;  // exponent all ones
      }
      poison = __any(any != 0);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) l += sc[b][r];
    u32x4 pf[4];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) pf[t][j] = pack_bf16(sc[t >> 1][8 * (t & 1) + 2 * j], sc[t >> 1][8 * (t & 1) + 2 * j + 1]);
    if (!poison) {
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = mma32_bf16(read_v(sV, t, d), pf[t], o[d]);
    } else {
      // values that are not finite as zeros, and, for every output, how many of them its
      // query sees (n) and their signs' sum (c): n of one sign give that infinity,
      // both signs or NaN (which has none) give NaN
#pragma unroll
      for (int d = 0; d < DB; ++d) {
        f16x n, c;
#pragma unroll
        for (int r = 0; r < 16; ++r) n[r] = c[r] = 0.f;
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const u32x4 v = read_v(sV, t, d);
          u32x4 fin, one, sign, sees;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            fin[j] = one[j] = sign[j] = sees[j] = 0;
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t x = v[j] >> (16 * e) & 0xffffu;
              const bool bad = (x & 0x7f80u) == 0x7f80u;
              fin[j] |= (bad ? 0u : x) << (16 * e);
              one[j] |= (bad ? 0x3f80u : 0u) << (16 * e);
              sign[j] |= ((x & 0x7fffu) == 0x7f80u ? 0x3f80u | (x & 0x8000u) : 0u) << (16 * e);
              sees[j] |= (key_of(t >> 1, 8 * (t & 1) + 2 * j + e) <= see ? 0x3f80u : 0u) << (16 * e);
            }
          }
          o[d] = mma32_bf16(fin, pf[t], o[d]);
          n = mma32_bf16(one, sees, n);
          c = mma32_bf16(sign, sees, c);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (n[r] > 0.f) o[d][r] += c[r] == n[r] ? INFINITY : c[r] == -n[r] ? -INFINITY : NAN;
      }
    }
  }
  // The compiler (ROCm 7.2) copied an accumulator at a loop's exit before its last
  // MFMA had written it; nothing may touch them until it has.
#pragma unroll
  for (int d = 0; d < DB; ++d) asm volatile("s_nop 15" : "+v"(o[d]));
  const int q = qw + l32;
  if (q >= lq) return;
  const auto rl = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  // queries that see no key: 0; a sum of 0 (every score -inf) gives NaN
  const float inv = 1.0f / (__uint_as_float(rl[0]) + __uint_as_float(rl[1]));
  const bool none = q + off < 0;
  uint16_t* y0 = a.O + (int64_t)(q_first + q) * a.ldo + head * HD + 4 * half;
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      uint16_t* yp = y0 + 32 * d + 8 * g;
      const uint32_t u0 = none ? 0u : pack_bf16(o[d][4 * g] * inv, o[d][4 * g + 1] * inv);
      const uint32_t u1 = none ? 0u : pack_bf16(o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv);
      if (a.vec) {
        *(uint2*)yp = make_uint2(u0, u1);
      } else {
        yp[0] = (uint16_t)u0;
        yp[1] = (uint16_t)(u0 >> 16);
        yp[2] = (uint16_t)u1;
        yp[3] = (uint16_t)(u1 >> 16);
      }
    }
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
  if (total_q > (int64_t)1 << 30 || total_k > (int64_t)1 << 30 || nseq > (int64_t)1 << 30) return DUO_ERR_UNSUPPORTED;
  if (nseq == 0 || total_q == 0) return DUO_OK;
  if (!Q || !O || !cu_q || (total_k > 0 && (!K || !V))) return DUO_ERR_INVALID_ARG;
  if (ldq % 8 || ldk % 8 || ldv % 8 || !aligned16(Q) || !aligned16(K) || !aligned16(V)) return DUO_ERR_UNSUPPORTED;
  // 128 queries per workgroup; 64 when that would leave CUs without their two
  // workgroups (512 in all)
  auto bound = [&](int64_t qb) { return total_q / qb + std::min(nseq, total_q); };
  const bool wide = (total_q / 128 + nseq / 2) * heads >= 512;
  const int64_t blocks = bound(wide ? 128 : 64);
  int64_t e = 1;
  while (e < 8 && kv_heads % (2 * e) == 0) e *= 2;
  const int64_t wgs = 8 * (kv_heads / e) * cdiv(blocks, 8 / e) * (heads / kv_heads);
  if (wgs > INT32_MAX) return DUO_ERR_UNSUPPORTED;
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  PackedArgs a;
  a.Q = (const uint16_t*)Q, a.K = (const uint16_t*)K, a.V = (const uint16_t*)V, a.O = (uint16_t*)O;
  a.ldq = ldq, a.ldk = ldk, a.ldv = ldv, a.ldo = ldo;
  a.cu_q = cu_q, a.cu_k = cu_k ? cu_k : cu_q;
  a.total_q = (int)total_q, a.total_k = (int)total_k, a.nseq = (int)nseq;
  a.kv_heads = (int)kv_heads, a.group = (int)(heads / kv_heads), a.blocks = (int)blocks;
  a.cexp = (float)(std::fabs(scale) * 1.4426950408889634);
  a.flip = scale < 0.0 ? 0x80008000u : 0u;
  a.vec = ldo % 4 == 0 && (reinterpret_cast<uintptr_t>(O) & 7) == 0;
  auto go = [&](auto kern, int nw) {
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(64 * nw), 0, (hipStream_t)stream, a);
  };
  if (head_dim == 128)
    wide ? go(packed_kernel<128, 4>, 4) : go(packed_kernel<128, 2>, 2);
  else
    wide ? go(packed_kernel<64, 4>, 4) : go(packed_kernel<64, 2>, 2);
  DUO_LAUNCH_CHECK();
  return DUO_OK;
}

}  // extern "C"
