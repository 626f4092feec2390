// Causal attention over packed sequences of different lengths, with grouped heads, in
// one pass over the keys with a running maximum and sum.
//
// One workgroup per (sequence, K/V head, block of 32 NW rows), a row being a query and one
// of the heads that read this K/V head, the heads of a query side by side: few queries
// fill a block all the same, and a wave's 32 rows end at nearly the same key.  Wave w owns
// rows 32 w .. 32 w + 31.  Everything is computed transposed, with v_mfma_f32_32x32x16_bf16
// (lane l holds row l % 32 of A and column l % 32 of B, the 8 consecutive k of half
// l / 32; accumulator element r sits at row 8 (r / 4) + 4 (l / 32) + r % 4, column
// l % 32):
//   S^T = K Q^T    a lane's 16 elements per block of 32 keys belong to one query;
//   O^T = V^T P^T  P^T's fragments are the lane's own probabilities, V^T's take the
//                  same keys from the row-major V tile with transposing LDS reads.
// K and V tiles of 64 keys stream global -> LDS directly, two buffers each; a wave's step is
// half a tile.
//
// Probabilities are taken relative to a running reference that is moved (and O and the
// sum with it) only when a score exceeds it by more than 8 in the exponent of two:
// they then stay below 2^8, which costs no accuracy in fp32 or bf16.  They are rounded to bf16
// for the product with V (the sum of them is not): a matrix instruction takes both operands in
// one type, and V's range is bf16's.  That is 2^-9 of each probability, of an output rounded
// to bf16 itself: against 64 bits the root mean square error of 2048 queries on 16384 keys is
// 0.0023 of the output's, and 0.0017 with probabilities in fp32.
//
// Few rows on long sequences: the keys of a block are split over workgroups, and a second
// launch joins the parts.
//
// Bound: MFMA issue beside the exponentials.  Heads of 128: one sequence of 16384 tokens, 64
// heads on 8, 3.9 to 4.1 ms (cards differ), 1080 to 1120 TFLOP/s (a large bf16 product reaches
// 1350); 8 of 2048, 32 heads, 0.35 ms, 780.  64 prompts of 256 tokens, 64 heads on 8, 175 to
// 196 us: of the 10 us of a block five are its start and end (two trips to memory one behind the
// other, the output), which the other workgroup of the CU covers in part.  Registers (236 of 256
// at two waves per SIMD) allow no third.  Blocks of 64 rows took 26.6 us for 1024 tokens with 32
// heads on 8 and 135 for 8 such sequences; of 128 24.4 and 103.  Heads of 64 have twice the
// exponentials per MFMA: 16384 tokens 2.4 ms, 930 TFLOP/s; 64 prompts of 256 tokens 99 us.
//
// Every workgroup looks for its sequence among all of them, 64 at a time: 1024 sequences of 16 tokens
// take 0.23 ms (their bytes 0.1), 8192 of them 7.9 (0.9).  Calls of many thousands of
// sequences are better made in pieces.
//
// Unseen keys get probability 0, and 0 times a value that is not finite would not be
// 0: in the steps where some query does not see some key such values enter as zeros,
// and the queries that do see them get them added at the end.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "dma.h"
#include "internal.h"
#include "mfma.h"
#include "pingpong.h"

#include "chunk_rows.h"

using namespace duo;
using namespace duo::pp;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 16) == 0; }

constexpr int NW = 4, QB = 32 * NW;  // waves of a workgroup, rows of a block

struct PackedArgs {
  const uint16_t *Q, *K, *V;
  uint16_t* O;
  int64_t ldq, ldk, ldv, ldo;
  const int32_t *cu_q, *cu_k;
  int total_q, total_k, nseq, kv_heads, group;
  uint32_t by_group;  // for by(): a row's query
  int by_shift;
  int blocks;  // bound of the blocks of rows of one K/V head
  float cexp;  // exp(s scale) = 2^(s cexp), with the queries' signs turned for a negative scale
  uint32_t flip;
  int vec;  // 16-byte stores of O
  // SPLIT: parts of a block's keys, and each part's outputs (rows x head_dim, not normalised)
  // and references and sums (rows x 2)
  int parts;
  float *po, *pml;
};

// n / group for 0 <= n < 2^31: with 2^(s-1) < group <= 2^s and by_group = ceil(2^(31+s) / group),
// by_group group is at most 2^s more than 2^(31+s), which never carries a quotient up.
__device__ inline int by(int n, const PackedArgs& a) { return (int)(__umulhi(2u * (uint32_t)n, a.by_group) >> a.by_shift); }

__device__ inline int cut(int v, int total) { return min(max(v, 0), total); }

// Of workgroup `id`: its K/V head, and which block of rows counted through all
// sequences.  Ids go round-robin over the XCDs: a K/V head lives on 8 / e of them, e =
// gcd(kv_heads, 8), which take its blocks in turn and share K and V in their L2.
__device__ inline bool place(int id, const PackedArgs& a, int* kv, int* block) {
  const int low = a.kv_heads & -a.kv_heads & 7, e = low ? low : 8, sh = 8 / e;
  const int x = id & 7, j = id >> 3;
  const int per = (a.blocks + sh - 1) / sh;  // blocks of one K/V head here
  *kv = j / per * e + x % e;
  *block = j % per * sh + x / e;
  return *kv < a.kv_heads && *block < a.blocks;
}

// A sequence's first rows and their numbers, and which block of it (the last one first).
struct Found {
  int q_first, lq, k_first, lk, qb;
};

// The sequence and the block within it of block b; false past the last.
__device__ inline bool find(const PackedArgs& a, int b, Found* f) {
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < a.nseq; s0 += 64) {
    const int s = min(s0 + lane, a.nseq - 1);
    const int q0 = cut(a.cu_q[s], a.total_q), q1 = cut(a.cu_q[s + 1], a.total_q);
    const int k0 = cut(a.cu_k[s], a.total_k), k1 = cut(a.cu_k[s + 1], a.total_k);
    const int n = s0 + lane < a.nseq ? (max(q1 - q0, 0) * a.group + QB - 1) / QB : 0;
    // running sum over the lanes: within rows of 16, then over the rows
    int up = n;
#define DUO_UP(o) up += __builtin_amdgcn_update_dpp(0, up, 0x110 + o, 0xf, 0xf, true)
    DUO_UP(1);
    DUO_UP(2);
    DUO_UP(4);
    DUO_UP(8);
#undef DUO_UP
    const int r0 = __builtin_amdgcn_readlane(up, 15), r1 = r0 + __builtin_amdgcn_readlane(up, 31);
    const int r2 = r1 + __builtin_amdgcn_readlane(up, 47);
    up += lane < 16 ? 0 : lane < 32 ? r0 : lane < 48 ? r1 : r2;
    const uint64_t past = __ballot(up > b);
    if (past) {
      const int l = __ffsll((unsigned long long)past) - 1;
      auto of = [&](int v) { return __builtin_amdgcn_readlane(v, l); };
      *f = Found{of(q0), of(q1 - q0), of(k0), max(of(k1 - k0), 0), of(up) - 1 - b};
      return true;
    }
    b -= __builtin_amdgcn_readlane(up, 63);
  }
  return false;
}

template <int HD, bool SPLIT>
__global__ __launch_bounds__(64 * NW, 2) void packed_kernel(PackedArgs a) {
  constexpr int KB = 64;                // keys per tile
  constexpr int CH = HD / 8;            // 16-byte chunks per key row
  constexpr int KS = HD / 16;           // MFMA steps over head_dim
  constexpr int DB = HD / 32;           // 32-wide blocks of the output row
  constexpr int TILE = KB * CH;         // chunks per operand tile
  constexpr int NL = TILE / (64 * NW);  // 16-byte loads per thread, operand and tile
  constexpr int RPL = 64 / CH;          // keys per wave-wide load
  __shared__ u32x4 sm[2][2][TILE];      // [buffer][K, V]
  int kv, block;
  Found f;
  const int part = SPLIT ? blockIdx.y : 0;
  if (!place(blockIdx.x, a, &kv, &block) || !find(a, block, &f)) return;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l32 = lane & 31, half = lane >> 5;
  const int q_first = f.q_first, lq = f.lq, k_first = f.k_first, lk = f.lk, qb = f.qb;
  const int off = lk - lq;              // query i sees keys j <= i + off
  // row r of the sequence and K/V head: query r / group, head r % group of its group
  const int rows = lq * a.group, row0 = qb * QB + 32 * wave, row = min(row0 + l32, rows - 1);
  const int q = by(row, a), head = kv * a.group + row - q * a.group;
  const int q_lo = by(row0, a), q_hi = by(min(row0 + 31, rows - 1), a);  // of this wave
  const uint16_t* const Kh = a.K + (int64_t)k_first * a.ldk + kv * HD;
  const uint16_t* const Vh = a.V + (int64_t)k_first * a.ldv + kv * HD;
  // chunk c of key row r sits at position kswz(r, c) (vswz) of its row: 16 consecutive
  // keys' chunks of a K fragment, and the four keys x 64 bytes that half a wave's
  // transposing read of V touches, cover the 64 banks once
  auto kswz = [](int key, int c) { return CH == 16 ? c ^ (key & 15) : c ^ ((key >> 1) & 7); };
  auto vswz = [](int key, int c) { return CH == 16 ? c ^ (4 * (key & 3)) : c ^ (4 * ((key >> 1) & 1)); };

  const int seen = by(min(qb * QB + QB - 1, rows - 1), a) + 1 + off;  // keys that the block's last query sees
  const int tiles = (seen + KB - 1) / KB;   // <= 0: none
  // this workgroup's: all of them, or a part that begins with an even one
  const int each = SPLIT ? max((tiles + a.parts - 1) / a.parts + 1 & ~1, 2) : 0;
  const int kb0 = part * each, nkb = SPLIT ? min(tiles, kb0 + each) : tiles;
  // this wave's part of tile kb of K (or V), keys past the last as the last
  auto issue = [&](const uint16_t* src, int64_t ld, int kb, const u32x4* dst, bool is_v) __attribute__((always_inline)) {
    const uint32_t to = __builtin_amdgcn_readfirstlane(lds_addr(dst + wave * NL * 64));
    const uint16_t* const tile = src + (int64_t)kb * KB * ld;
    const int left = lk - 1 - kb * KB;  // the last key's place in the tile
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int key = (wave * NL + i) * RPL + lane / CH, p = lane % CH;
      const int row = left >= KB ? key : min(key, left);
      const int c = is_v ? vswz(key, p) : kswz(key, p);
      dma16(tile, (uint32_t)row * (uint32_t)(ld * 2) + 16 * c, to + i * 1024);
    }
  };

  // the first keys and the queries are on their way together
  if (nkb > kb0) issue(Kh, a.ldk, kb0, sm[0][0], false);
  u32x4 qa[KS];
  {
    const uint16_t* at = a.Q + (int64_t)(q_first + q) * a.ldq + head * HD;
#pragma unroll
    for (int c = 0; c < KS; ++c) qa[c] = *(const u32x4*)(at + 8 * (2 * c + half));
#pragma unroll
    for (int c = 0; c < KS; ++c) {
      asm volatile("" : "+v"(qa[c]));  // waited for here, and not behind the loads that follow
#pragma unroll
      for (int j = 0; j < 4; ++j) qa[c][j] ^= a.flip;
    }
  }

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
  // Steps of 32 keys, two per tile.  This wave: steps of which its queries see a key, and of
  // which they see every key.
  const int nu = row0 < rows && q_hi + off >= 0 ? min((q_hi + off) / 32 + 1, 2 * nkb) : 0;  // up to step nu
  const int u0 = 2 * kb0;
  const int nfull = max((q_lo + off + 1) / 32, 0);
  auto key_of = [&](int r) { return 8 * (r >> 2) + 4 * half + (r & 3); };

  f16x sa, sb;  // scores of an even and of an odd step
  u32x4 pf[2];  // probabilities of a step
  auto k_rows = [&](int u) { return (const u32x4*)sm[u >> 1 & 1][0] + (u & 1) * 32 * CH; };
  auto v_rows = [&](int u) { return (const uint8_t*)sm[u >> 1 & 1][1] + (u & 1) * 32 * HD * 2; };
  auto read_k = [&](const u32x4* sK, int c) { return sK[l32 * CH + kswz(l32, 2 * c + half)]; };
  auto score = [&](int u, f16x& sc) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
    for (int c = 0; c < KS; ++c) sc = mma32_bf16(read_k(k_rows(u), c), qa[c], sc);
  };
  // a new reference where the step's scores leave the old one's range: the factor of what is
  // relative to the old one (1 elsewhere), and whether any lane has one
  auto refer = [&](const f16x& sc, float* f) __attribute__((always_inline)) {
    float mt = sc[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mt = fmaxf(mt, sc[r]);
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
    mt = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
    const bool up = mt > m && !(mt * a.cexp <= mc + 8.f);
    if (!__any(up)) return false;
    const float mcn = up ? mt * a.cexp : mc;
    *f = up ? m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - mcn) : 1.f;
    m = up ? mt : m;
    mc = mcn;
    l *= *f;
    return true;
  };
  auto scale_o = [&](float f) __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < DB; ++d) asm volatile("s_nop 15" : "+v"(o[d]));  // the last products have been written
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] *= f;
  };
  // probabilities of a step, and their sum
  auto probabilities = [&](const f16x& sc, u32x4 (&p)[2]) __attribute__((always_inline)) {
    const float base = m == -INFINITY ? 0.f : mc;
    float sum = 0.f;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[8 * t + 2 * j], a.cexp, -base));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[8 * t + 2 * j + 1], a.cexp, -base));
        sum += p0 + p1;
        p[t][j] = pack_bf16(p0, p1);
      }
    return sum;
  };
  // O += V^T P^T of step u
  typedef short s16v2 __attribute__((ext_vector_type(2)));
  typedef unsigned short u16v2 __attribute__((ext_vector_type(2)));
  bool poison = false;
  auto add = [&](int u) __attribute__((always_inline)) {
    const uint8_t* sV = v_rows(u);
    u32x4 v[2][DB];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int d = 0; d < DB; ++d) v[t][d] = read_v(sV, t, d);
    if (u >= nfull) {
      // some query does not see some key: are there numbers that are not finite?  As 16-bit
      // integers those are the largest, signed for one sign and unsigned for the other.
      s16v2 ms[4] = {};
      u16v2 mu[4] = {};
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s16v2 x;
            u16v2 y;
            const uint32_t w = v[t][d][j];
            __builtin_memcpy(&x, &w, 4);
            __builtin_memcpy(&y, &w, 4);
            ms[j] = __builtin_elementwise_max(ms[j], x);
            mu[j] = __builtin_elementwise_max(mu[j], y);
          }
      const s16v2 most_s = __builtin_elementwise_max(__builtin_elementwise_max(ms[0], ms[1]), __builtin_elementwise_max(ms[2], ms[3]));
      const u16v2 most_u = __builtin_elementwise_max(__builtin_elementwise_max(mu[0], mu[1]), __builtin_elementwise_max(mu[2], mu[3]));
      if (__any(most_s[0] >= 0x7f80 || most_s[1] >= 0x7f80 || most_u[0] >= 0xff80 || most_u[1] >= 0xff80)) {
        poison = true;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t w = v[t][d][j];
              const uint32_t lo = (w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u, hi = (w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u;
              v[t][d][j] = w & ~(lo | hi);
            }
      }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int d = 0; d < DB; ++d) o[d] = mma32_bf16(v[t][d], pf[t], o[d]);
  };
  // Step u's probabilities, the values of the step before and the scores of the next are
  // independent of each other.  Where all three are there and nothing is masked they are
  // dealt out evenly: MFMAs of the one, LDS reads and vector instructions of the others.
  auto fast = [&](auto place, f16x& sc, f16x& sn) __attribute__((always_inline)) {
    constexpr int P = decltype(place)::value;  // the step's place in two tiles, as its LDS buffers go by it
    const float base = mc;
    const u32x4* sK = k_rows(P + 1);
    const uint8_t* sV = v_rows(P + 3);
    u32x4 pn[2];
    float ls[2] = {0.f, 0.f}, most = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sn[r] = 0.f;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int r = 8 * t + 2 * j;
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[r], a.cexp, -base));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[r + 1], a.cexp, -base));
        ls[0] += p0;
        ls[1] += p1;
        most = fmaxf(most, fmaxf(p0, p1));
        pn[t][j] = pack_bf16(p0, p1);
      }
#pragma unroll
      for (int i = 0; i < KS / 2; ++i) {
        const int c = t * (KS / 2) + i;
        sn = mma32_bf16(read_k(sK, c), qa[c], sn);
        if (i < DB) o[i] = mma32_bf16(read_v(sV, t, i), pf[t], o[i]);
      }
    }
    float sum = ls[0] + ls[1];
    asm volatile("" : "+v"(pn[0]), "+v"(pn[1]), "+v"(sum), "+v"(most));  // computed here, not where they are used
    __builtin_amdgcn_sched_group_barrier(0x100, 6, 0);
#pragma unroll
    for (int i = 0; i < DB + KS / 2; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, HD == 128 ? 4 : 8, 0);
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, HD == 128 ? 4 : 8, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    // scores that leave the reference's range (or have none yet): once more, with another
    if (__any(most > 256.f || m == -INFINITY)) {
      float f = 1.f;
      if (refer(sc, &f)) scale_o(f);
      sum = probabilities(sc, pn);
    }
    l += sum;
    pf[0] = pn[0];
    pf[1] = pn[1];
  };
  auto slow = [&](int u, f16x& sc, f16x& sn) __attribute__((always_inline)) {
    if (u > u0 && u <= nu) add(u - 1);
    if (u < nu) {
      const int see = q + off - u * 32;
      if (u >= nfull)
#pragma unroll
        for (int r = 0; r < 16; ++r) sc[r] = key_of(r) > see ? -INFINITY : sc[r];
      float f;
      if (refer(sc, &f) && u > u0) scale_o(f);
      l += probabilities(sc, pf);
      if (u + 1 < nu) score(u + 1, sn);
    }
  };

  if (nkb > kb0) {
    issue(Kh, a.ldk, min(kb0 + 1, nkb - 1), sm[1][0], false);
    issue(Vh, a.ldv, kb0, sm[0][1], true);
    wait_vm<2 * NL>();
    lds_barrier();
    if (nu > u0) score(u0, sa);
  }
  // K of the next tile and V of this one have landed, and every wave is done with K of
  // this one and V of the one before, whose places the next ones take
  auto turn = [&](int kb) __attribute__((always_inline)) {
    wait_vm<0>();
    lds_barrier();
    if (kb + 2 < nkb) issue(Kh, a.ldk, kb + 2, sm[kb & 1][0], false);
    if (kb + 1 < nkb) issue(Vh, a.ldv, kb + 1, sm[(kb + 1) & 1][1], true);
  };
  for (int kb = kb0; kb < nkb;) {
    slow(2 * kb, sa, sb);
    turn(kb);
    slow(2 * kb + 1, sb, sa);
    // two tiles at a time, the odd one first, so that places in LDS are known when compiled
    for (++kb; (kb & 1) && 2 * kb + 4 < nu && 2 * kb + 3 < nfull; kb += 2) {
      fast(std::integral_constant<int, 2>{}, sa, sb);
      turn(kb);
      fast(std::integral_constant<int, 3>{}, sb, sa);
      fast(std::integral_constant<int, 0>{}, sa, sb);
      turn(kb + 1);
      fast(std::integral_constant<int, 1>{}, sb, sa);
    }
  }
  if (nu > u0 && nu == 2 * nkb) add(nu - 1);
  // The compiler (ROCm 7.2) copied an accumulator at a loop's exit before its last
  // MFMA had written it; nothing may touch them until it has.
#pragma unroll
  for (int d = 0; d < DB; ++d) asm volatile("s_nop 15" : "+v"(o[d]));
  if (poison) {
    // what every query sees of the numbers left out (infinities and NaN add up as they do)
#pragma unroll 1
    for (int j = max(nfull, u0) * 32; j < min(nu * 32, lk); ++j) {
      const uint16_t* v = Vh + (int64_t)j * a.ldv + 4 * half;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float x = bf16_bits_to_f32(v[32 * d + 8 * (r >> 2) + (r & 3)]);
          o[d][r] += j <= q + off && !(fabsf(x) < INFINITY) ? x : 0.f;
        }
    }
  }
  const auto rl = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
  if constexpr (SPLIT) {
    const int64_t at = (((int64_t)kv * a.blocks + block) * a.parts + part) * QB + 32 * wave + l32;
    if (half == 0) *(float2*)(a.pml + 2 * at) = make_float2(mc, __uint_as_float(rl[0]) + __uint_as_float(rl[1]));
    float* y = a.po + at * HD + 4 * half;
    if (nu > u0)
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          *(f4*)(y + 32 * d + 8 * g) = f4{o[d][4 * g], o[d][4 * g + 1], o[d][4 * g + 2], o[d][4 * g + 3]};
    return;
  }
  // queries that see no key: 0; a sum of 0 (every score -inf) gives NaN
  const float inv = q + off < 0 ? 0.f : 1.0f / (__uint_as_float(rl[0]) + __uint_as_float(rl[1]));
  uint2 y[DB][4];
#pragma unroll
  for (int d = 0; d < DB; ++d)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      y[d][g].x = pack_bf16(o[d][4 * g] * inv, o[d][4 * g + 1] * inv);
      y[d][g].y = pack_bf16(o[d][4 * g + 2] * inv, o[d][4 * g + 3] * inv);
    }
  if (a.vec) {
    // through this wave's part of LDS, where the last K tiles were (every wave was done with
    // them at the last turn), so that a row is written at once, 16 bytes per lane; chunk c of
    // row r at c ^ (r % CH)
    uint8_t* const st = (uint8_t*)sm[wave / (NW / 2)][0] + wave % (NW / 2) * (32 * HD * 2);
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *(uint2*)(st + l32 * HD * 2 + ((4 * d + g) ^ (l32 & (CH - 1))) * 16 + 8 * half) = y[d][g];
    wait_lds<0>();
    uint16_t* const O0 = a.O + (int64_t)q_first * a.ldo + 8 * (lane % CH);
#pragma unroll
    for (int i = 0; i < 32 / RPL; ++i) {
      const int r = i * RPL + lane / CH, qr = by(row0 + r, a), h = kv * a.group + (row0 + r) - qr * a.group;
      const u32x4 v = *(const u32x4*)(st + r * HD * 2 + (lane % CH ^ (r & (CH - 1))) * 16);
      if (row0 + r < rows) *(u32x4*)(O0 + qr * a.ldo + h * HD) = v;
    }
  } else if (row0 + l32 < rows) {
    uint16_t* y0 = a.O + (int64_t)(q_first + q) * a.ldo + head * HD + 4 * half;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        uint16_t* yp = y0 + 32 * d + 8 * g;
        yp[0] = (uint16_t)y[d][g].x;
        yp[1] = (uint16_t)(y[d][g].x >> 16);
        yp[2] = (uint16_t)y[d][g].y;
        yp[3] = (uint16_t)(y[d][g].y >> 16);
      }
  }
}

// Joins the parts of a block's rows: HD / 4 threads per row, blockIdx.y counts the rows of a
// block by the 1024 / HD that a workgroup takes.
template <int HD>
__global__ __launch_bounds__(256) void packed_join_kernel(PackedArgs a) {
  constexpr int T = HD / 4;
  int kv, block;
  Found f;
  if (!place(blockIdx.x, a, &kv, &block) || !find(a, block, &f)) return;
  const int local = blockIdx.y * (256 / T) + threadIdx.x / T, row = f.qb * QB + local, d = threadIdx.x % T * 4;
  if (row >= f.lq * a.group) return;
  const int q = by(row, a), head = kv * a.group + row - q * a.group;
  const int64_t at = ((int64_t)kv * a.blocks + block) * a.parts * QB + local;
  float top = -INFINITY;
#pragma unroll 4
  for (int i = 0; i < a.parts; ++i) top = fmaxf(top, a.pml[2 * (at + (int64_t)i * QB)]);
  float sum = 0.f;
  f4 y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = 0; i < a.parts; ++i) {
    const float2 ml = *(const float2*)(a.pml + 2 * (at + (int64_t)i * QB));
    if (ml.x == -INFINITY && ml.y == 0.f) continue;  // nothing seen, and nothing written
    const float w = ml.x == -INFINITY ? ml.y : __builtin_amdgcn_exp2f(ml.x - top);
    sum += w * ml.y;
    y += *(const f4*)(a.po + (at + (int64_t)i * QB) * HD + d) * w;
  }
  const bool none = q + f.lk - f.lq < 0;
  const uint2 two = none ? make_uint2(0, 0) : make_uint2(pack_bf16(y[0] / sum, y[1] / sum), pack_bf16(y[2] / sum, y[3] / sum));
  uint16_t* const o = a.O + (int64_t)(f.q_first + q) * a.ldo + head * HD + d;
  if (a.vec) {
    *(uint2*)o = two;
  } else {
    o[0] = (uint16_t)two.x, o[1] = (uint16_t)(two.x >> 16);
    o[2] = (uint16_t)two.y, o[3] = (uint16_t)(two.y >> 16);
  }
}

// How a call is cut: a bound of the blocks of a K/V head, parts of their keys.
struct Plan {
  int64_t blocks, parts;
};
Plan packed_plan(int64_t total_q, int64_t total_k, int64_t nseq, int64_t group, int64_t kv_heads) {
  const int64_t blocks = total_q * group / QB + std::min(nseq, total_q), wgs = blocks * kv_heads;
  // Few rows on long sequences leave most CUs idle, so their keys are split too: as many
  // parts as fill the CUs (two workgroups on each), of 512 keys at least (on average over the
  // sequences).  One query on 16384 keys, 64 heads on 8: 238 us whole, 33 split, 44 with
  // parts of 256 keys; 256 queries there 261 and 166; where nothing is split for shortness, 512
  // queries on 512 keys, 32 heads on 8: 15 us, and 20 in parts of 256.
  const int64_t parts = std::min<int64_t>({512 / wgs, total_k / nseq / 512, 64});
  return {blocks, parts >= 2 ? parts : 1};
}

// Workgroups of rows_kernel, a multiple of eight: no more than the smallest shares of all that the
// sizes allow.
int64_t rows_wgs(int64_t total_q, int64_t nseq, int64_t group, int64_t kv_heads, int64_t max_len) {
  const int64_t nsub = cdiv(group, kRowsQB), qpb = kRowsQB / cdiv(group, nsub);
  const double blocks = (double)(kv_heads * nsub) * (double)(total_q / qpb + std::min(nseq, total_q));
  const double shares = blocks * (double)(max_len + qpb + kRowsCost) / kRowsMin + 1;
  return shares < kRowsWg ? rup((int64_t)shares, 8) : kRowsWg;
}

}  // namespace

namespace duo {

// How many sequences may have their rows made of codes before (0: none), and the tiles and bytes for them.
struct Made {
  int64_t seqs, tiles, flags, bytes;
  Made(int32_t format, int64_t total_q, int64_t nseq, int64_t group, int64_t kv_heads, int64_t head_dim, int64_t max_len) {
    seqs = format == DUO_KV_BF16 || nseq > 64 ? 0 : std::min(nseq, total_q * group / (kRowsMany + 1));
    tiles = cdiv(max_len, 64);
    if (seqs * tiles * kv_heads > ((int64_t)1 << 30) / (64 * 4 * head_dim)) seqs = 0;  // a workspace of 1 GiB at most
    flags = rup(seqs * tiles * kv_heads, 1024);
    bytes = seqs ? (int64_t)align_up(flags) + seqs * tiles * kv_heads * 64 * 4 * head_dim : 0;
  }
};

size_t chunk_rows_ws_bytes(int32_t format, int64_t total_q, int64_t nseq, int64_t heads, int64_t kv_heads, int64_t head_dim,
                           int64_t max_len) {
  const int64_t group = heads / kv_heads, wgs = rows_wgs(total_q, nseq, group, kv_heads, max_len);
  return align_up(wgs * sizeof(RowsTask)) + align_up((size_t)(2 * wgs * rows_part((int)head_dim)) * sizeof(float)) +
         align_up(Made(format, total_q, nseq, group, kv_heads, head_dim, max_len).bytes);
}

duo_status chunk_rows_run(const ChunkCall& c, int64_t least, void* ws, hipStream_t s) {
  RowsArgs a = {};
  a.Q = (const uint16_t*)c.Q, a.O = (uint16_t*)c.O;
  a.ldq = c.ldq, a.ldo = c.ldo;
  a.kv = c.geo;
  a.table = c.table, a.ldt = c.ldt, a.lens = c.lens, a.cu_q = c.cu_q;
  a.total_q = (int)c.total_q, a.nseq = (int)c.nseq, a.max_len = (int)c.max_len;
  a.group = (int)(c.heads / c.geo.heads);
  a.nsub = (int)cdiv(a.group, kRowsQB), a.hg = (int)cdiv(a.group, a.nsub), a.qpb = kRowsQB / a.hg;
  while ((1 << a.by_shift) < a.hg) ++a.by_shift;
  a.by_hg = (uint32_t)((((uint64_t)1 << (31 + a.by_shift)) + a.hg - 1) / a.hg);
  a.window = c.window, a.sinks = c.sinks;
  a.per = (int)cdiv(c.nseq, 64);
  a.least = least, a.most = INT64_MAX, a.over = kRowsMany;
  a.flip = c.flip;
  a.vec = c.ldo % 8 == 0 && aligned16(c.O);
  const int64_t wgs = rows_wgs(c.total_q, c.nseq, a.group, c.geo.heads, c.max_len);
  a.deal = wgs % (c.geo.heads * a.nsub) == 0 ? (int)(wgs / (c.geo.heads * a.nsub)) : 0;
  a.tasks = (RowsTask*)ws;
  a.parts = (float*)((uint8_t*)ws + align_up(wgs * sizeof(RowsTask)));
  return kv_by_format(c.cache, [&](auto fmt, auto dim) -> duo_status {
    constexpr int FMT = decltype(fmt)::value, HD = decltype(dim)::value;
    auto go = [&](auto f, const RowsArgs& r) -> duo_status {
      constexpr int F = decltype(f)::value, lds = RowsGeo<F, HD>::LDS;
      const auto kern = rows_kernel<F, HD>;
      if (duo_status st = set_max_lds((const void*)kern, lds); st != DUO_OK) return st;
      hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), lds, s, r);
      DUO_LAUNCH_CHECK();
      if (wgs > 1) {
        hipLaunchKernelGGL(HIP_KERNEL_NAME(rows_join_kernel<HD, F == DUO_KV_I4>), dim3((unsigned)wgs, kRowsQB * HD / 1024),
                           dim3(256), 0, s, r);
        DUO_LAUNCH_CHECK();
      }
      return DUO_OK;
    };
    // numbers in fp16 are 2^6 of themselves; never 0, as above
    a.cexp = FMT == DUO_KV_BF16 ? c.cexp : std::max(std::ldexp(c.cexp, -kRowsBoost), 1.4e-45f);
    if constexpr (FMT != DUO_KV_BF16) {
      const Made made(FMT, c.total_q, c.nseq, a.group, c.geo.heads, HD, c.max_len);
      if (made.seqs && c.max_q * a.group > kRowsMany) {
        uint8_t* const flags = (uint8_t*)ws + align_up(wgs * sizeof(RowsTask)) + align_up((size_t)(2 * wgs * rows_part(HD)) * sizeof(float));
        uint8_t* const rows = flags + align_up(made.flags);
        a.flags = flags, a.nflags = (int)made.flags, a.made_tiles = (int)made.tiles;
        hipLaunchKernelGGL(HIP_KERNEL_NAME(rows_make_kernel<FMT, HD>),
                           dim3((unsigned)made.tiles, (unsigned)c.geo.heads, (unsigned)made.seqs), dim3(256), 0, s, a, rows, flags);
        DUO_LAUNCH_CHECK();
        RowsArgs r = a;
        r.least = kRowsMany;
        r.kv.data = rows, r.kv.pages = made.seqs * made.tiles, r.kv.block = 64 * 4 * HD, r.kv.shift = 6;
        if (duo_status st = go(std::integral_constant<int, kKvMade>{}, r); st != DUO_OK) return st;
      }
    }
    return go(fmt, a);
  });
}

}  // namespace duo

extern "C" {

size_t duo_attention_packed_workspace_size(int64_t total_q, int64_t total_k, int64_t nseq, int64_t heads,
                                           int64_t kv_heads, int64_t head_dim) {
  if (total_q < 1 || total_k < 1 || nseq < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads ||
      (head_dim != 64 && head_dim != 128) || heads > 65535 || total_q * (heads / kv_heads) > INT32_MAX / 2)
    return 0;
  const Plan p = packed_plan(total_q, total_k, nseq, heads / kv_heads, kv_heads);
  if (p.parts == 1) return 0;
  return align_up((size_t)(p.blocks * kv_heads * p.parts * QB * (head_dim + 2)) * sizeof(float));
}

duo_status duo_attention_packed(const void* Q, int64_t ldq, const void* K, int64_t ldk, const void* V, int64_t ldv,
                                const int32_t* cu_q, int64_t total_q, const int32_t* cu_k, int64_t total_k,
                                int64_t nseq, int64_t heads, int64_t kv_heads, int64_t head_dim, double scale, void* O,
                                int64_t ldo, void* ws, size_t ws_bytes, void* stream) {
  if (nseq < 0 || total_q < 0 || total_k < 0 || heads < 1 || kv_heads < 1 || head_dim < 1 || heads > 65535 ||
      kv_heads > heads || heads % kv_heads || !std::isfinite(scale))
    return DUO_ERR_INVALID_ARG;
  if (ldq < heads * head_dim || ldo < heads * head_dim || ldk < kv_heads * head_dim || ldv < kv_heads * head_dim)
    return DUO_ERR_INVALID_ARG;
  if (!cu_k && total_k != total_q) return DUO_ERR_INVALID_ARG;
  if (head_dim != 64 && head_dim != 128) return DUO_ERR_UNSUPPORTED;
  if (ldk >= 1 << 24 || ldv >= 1 << 24) return DUO_ERR_UNSUPPORTED;  // a tile within 2^31 bytes
  if (total_q > (int64_t)1 << 30 || total_k > (int64_t)1 << 30 || nseq > (int64_t)1 << 30) return DUO_ERR_UNSUPPORTED;
  if (nseq == 0 || total_q == 0) return DUO_OK;
  if (!Q || !O || !cu_q || (total_k > 0 && (!K || !V))) return DUO_ERR_INVALID_ARG;
  if (ldq % 8 || ldk % 8 || ldv % 8 || !aligned16(Q) || !aligned16(K) || !aligned16(V)) return DUO_ERR_UNSUPPORTED;
  const int64_t group = heads / kv_heads;
  if (total_q * group > INT32_MAX / 2) return DUO_ERR_UNSUPPORTED;
  const size_t need = duo_attention_packed_workspace_size(total_q, total_k, nseq, heads, kv_heads, head_dim);
  if (need && (!ws || ws_bytes < need || reinterpret_cast<uintptr_t>(ws) % kAlign)) return DUO_ERR_WORKSPACE;
  const Plan plan = packed_plan(total_q, total_k, nseq, group, kv_heads);
  const int64_t blocks = plan.blocks;
  int64_t e = 1;
  while (e < 8 && kv_heads % (2 * e) == 0) e *= 2;
  const int64_t wgs = 8 * (kv_heads / e) * cdiv(blocks, 8 / e);
  if (wgs > kMaxGrid) return DUO_ERR_UNSUPPORTED;
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  PackedArgs a;
  a.Q = (const uint16_t*)Q, a.K = (const uint16_t*)K, a.V = (const uint16_t*)V, a.O = (uint16_t*)O;
  a.ldq = ldq, a.ldk = ldk, a.ldv = ldv, a.ldo = ldo;
  a.cu_q = cu_q, a.cu_k = cu_k ? cu_k : cu_q;
  a.total_q = (int)total_q, a.total_k = (int)total_k, a.nseq = (int)nseq;
  a.kv_heads = (int)kv_heads, a.group = (int)group, a.blocks = (int)blocks;
  a.by_shift = 0;
  while ((int64_t)1 << a.by_shift < group) ++a.by_shift;
  a.by_group = (uint32_t)((((uint64_t)1 << (31 + a.by_shift)) + group - 1) / group);
  // never 0: the scores of keys that are not seen, -inf, have to stay that
  a.cexp = std::max((float)(std::fabs(scale) * 1.4426950408889634), 1.4e-45f);
  a.flip = scale < 0.0 ? 0x80008000u : 0u;
  a.vec = ldo % 8 == 0 && aligned16(O);
  a.parts = (int)plan.parts;
  const int64_t rows = blocks * kv_heads * plan.parts * QB;
  a.po = (float*)ws;
  a.pml = a.po + (need ? rows * head_dim : 0);
  const hipStream_t st = (hipStream_t)stream;
  auto go = [&](auto hd) -> duo_status {
    constexpr int HD = decltype(hd)::value;
    const dim3 grid((unsigned)wgs, (unsigned)plan.parts);
    if (plan.parts > 1) {
      hipLaunchKernelGGL(HIP_KERNEL_NAME(packed_kernel<HD, true>), grid, dim3(64 * NW), 0, st, a);
      DUO_LAUNCH_CHECK();
      hipLaunchKernelGGL(packed_join_kernel<HD>, dim3((unsigned)wgs, QB * HD / 1024), dim3(256), 0, st, a);
    } else {
      hipLaunchKernelGGL(HIP_KERNEL_NAME(packed_kernel<HD, false>), grid, dim3(64 * NW), 0, st, a);
    }
    DUO_LAUNCH_CHECK();
    return DUO_OK;
  };
  return head_dim == 128 ? go(std::integral_constant<int, 128>{}) : go(std::integral_constant<int, 64>{});
}

}  // extern "C"
