// Attention of new tokens over the paged cache where a sequence has many rows: the kernel of
// chunks (duo_attention_chunk), by whose side the paged kernel does the sequences of few rows.
// Included by the one file that compiles it, behind dma.h, pingpong.h and mfma.h.
//
// A block is up to 128 rows of one sequence and K/V head, a row being a new token and one of the
// heads that read this K/V head, the heads of a token side by side; wave w owns the rows 32 w
// .. 32 w + 31.  As in the packed kernel everything is computed transposed on 32-wide MFMA tiles
// (S^T = K Q^T, O^T = V^T P^T with P^T's fragments the lane's own probabilities and V^T's from
// transposing LDS reads), in steps of 32 keys, with a running reference that moves only when
// a score exceeds it by a factor of 2^8, and probabilities rounded to bf16 for the product with V.
//
// Tiles are 64 keys of the pages: a wave brings 16 of them (a run), which lie in one page whatever
// its size.  A block's tiles are those of the sinks, then those from its first query's window on.  Keys
// behind the end are copies of the last one.  In 16 bits rows go global -> LDS directly.
//
// In 8 and 4 bits the codes do, to a place of the wave's own, and a turn later the wave makes
// numbers of them in the tile that all waves read: once for 128 rows, where the paged kernel, which
// multiplies the codes themselves, pays for scales in every product.  The numbers are fp16 and so is
// everything that they meet: a code of 4 bits times a scale (three bits times eight) is exact in it, one
// of 8 bits is rounded to 2^-11 of itself (bf16 would cost 2^-8: an error of the output of 0.0031 and, in
// 4 bits, 0.0048 of its root mean square, where the plain form has 0.0017).  fp16's range is made to
// do by powers of two: a key whose largest number is outside 2^-2 .. 2^8 is brought to 2^7, and its
// scores take the power back; a row of Q likewise; and a token's values (small ones to 2^-2), whose power goes into the
// exponent of its probabilities (the running reference is then one of p |V|, not of p).  The sum of
// the p then lies anywhere beside the reference (values reach from 2^-126 to 2^127), and gets a power of its own
// where it is far from it.  Values are in units of a power of two that the first two tiles' largest one says; results do not
// go by it, nor by keys that no query of the block sees.  The steps that are dealt out go without all of that: a tile with
// a key outside 2^-2 .. 2^8, a token of values outside 2^-6 .. 2^4 (or such a range around the first tiles') or one of zeros
// takes others, of about twice the time (where most tokens of values have powers: 128 on 16384, 64 heads on 8, 126 us and
// 231).  Sequences of very many rows have their numbers made once, by a launch before, into the
// workspace (rows_make_kernel): 2048 tokens on 16384, 64 heads on 8, 1362 us without in 8 bits, 1110 with
// it; 320 on 8192, 32 on 8 (1280 rows), 104 and 101, on 65536 558 and 496; with 1024 rows it gains
// nothing up to 32768.  If there is one among them that needs a power (values from 2^5 on), all of that is left, for all
// sequences, and they are done from the codes as the others are (2048 tokens there 1490 us).  What is lost: bits of groups of 32 channels whose scale is below 2^-18 of the token's largest number, and
// of probabilities in fp16: up to 2^-25 beside 2^6 and more of the reference's token, which is, with values in
// [2^-2, 2^8), up to 2^-20 of the largest p |V| of all channels for a key (so a token with a number of 2^27 in one group and
// ordinary ones in another takes bits of the others' part in both).
//
// A sequence with more blocks than there are workgroups gives each the same number of them, whole, the long
// ones dealt out against the short ones: all workgroups of an XCD then read one head's keys at
// the same time, which keeps them in its L2 (2048 tokens on 16384, 64 heads on 8: 982 us, 1086 without; 987 to 1022 on
// other cards).  All other
// blocks cost what they have of keys, and something for their start and end; their count
// is cut into equal shares, one per workgroup, neighbours on one XCD.  A share's end that lies
// near a block's end is moved there; a block in several shares is joined by a second launch.  All of
// that follows from the lengths, on the device: no atomics, equal results every time.
#pragma once

#include "cache.h"

namespace duo {

using namespace pp;

constexpr int kRowsQB = 128;     // rows of a block
constexpr int kRowsWg = 512;     // workgroups at most: two on each CU
constexpr int kRowsCost = 128;   // what a block's start and end cost, in keys (256: 0 to 2 us more in short calls)
constexpr int kRowsMin = 512;    // smallest share, in keys: 16 tokens on 16384, 64 heads on 8, 60 us, 98 with 256
constexpr int kRowsMany = 1279;  // sequences with more rows than this have their numbers made of codes before (if all fit 1 GiB)
constexpr int kRowsSnap = 512;   // a share's end moves to a block's end that is no further than this
// Tokens are 2^30 at most: a place behind all of a block, and a window that hides none.
constexpr int kRowsAll = INT32_MAX, kRowsBack = 1 << 30;

struct RowsArgs {
  const uint16_t* Q;
  uint16_t* O;
  int64_t ldq, ldo;
  KvGeo kv;
  const int32_t* table;
  int64_t ldt;
  const int32_t *lens, *cu_q;
  int total_q, nseq, max_len, group;
  int hg, nsub, qpb;  // heads of a block and such parts of a group, queries of a block
  uint32_t by_hg;     // see by()
  int by_shift;
  int window, sinks;
  int per;        // sequences per bucket of the count
  int deal;       // blocks of one head that a round of all workgroups takes: 0 where heads do not divide them
  int64_t least, most;  // sequences with more rows than least, and no more than most, are done here
  // Rows made of codes: the sequences with more than `over` rows, one behind the other, made_tiles tiles
  // for each, and what says of some of them that their numbers do not fit fp16 as they are (none: NULL).
  int64_t over;
  const uint8_t* flags;
  int nflags, made_tiles;  // nflags: a multiple of 1024
  float cexp;     // exp(s scale) = 2^(s cexp), with the queries' signs turned for a negative scale
  uint32_t flip;
  int vec;        // 16-byte stores of O
  struct RowsTask* tasks;
  float* parts;  // two places per share
};

// Of a part, in floats: outputs (rows x head_dim, not normalised), references and sums.
constexpr int64_t rows_part(int hd) { return kRowsQB * (int64_t)(hd + 2); }

// A block that begins in a share and ends in another one.
struct RowsTask {
  int parts, q0, head0, heads, rows, pos0;
};

// n / hg for 0 <= n < 2^31: by_hg = ceil(2^(31+s) / hg) with 2^(s-1) < hg <= 2^s
__device__ inline int by(int n, const RowsArgs& a) { return (int)(__umulhi(2u * (uint32_t)n, a.by_hg) >> a.by_shift); }

__device__ inline uint64_t rows_div(uint64_t a, uint64_t b) { return (a | b) >> 32 ? a / b : (uint32_t)a / (uint32_t)b; }

// A sequence as the count sees it: block n costs min(first + (n + 1) qpb, most) keys, and kRowsCost.
struct RowsSeq {
  int q0, lq, len;
  int nb, dealt;            // blocks of a head that are counted: the first ones; those behind them are dealt out
  int first, most, linear;  // tokens before the first new one; most keys of a block; blocks below it

  RowsSeq() = default;
  __device__ RowsSeq(const RowsArgs& a, int s) {
    const bool in = s < a.nseq;
    const int x = in ? min(max(a.cu_q[s], 0), a.total_q) : 0, y = in ? min(max(a.cu_q[s + 1], 0), a.total_q) : 0;
    q0 = x, lq = max(y - x, 0), len = in ? min(max(a.lens[s], 0), a.max_len) : 0;
    const int64_t rows = (int64_t)lq * a.group;
    nb = rows > a.least && rows <= a.most ? (lq + a.qpb - 1) / a.qpb : 0;
    dealt = a.deal ? nb / a.deal * a.deal : 0;
    nb -= dealt;
    first = max(len - lq, 0);
    most = a.window ? (int)min((int64_t)a.window + a.sinks + a.qpb + 192, (int64_t)INT32_MAX - 4096) : INT32_MAX;
    linear = most < first ? 0 : min((most - first) / a.qpb, nb);
  }
  __device__ int cost(int n, const RowsArgs& a) const {
    return (n < linear ? first + (n + 1) * a.qpb : most) + kRowsCost;
  }
  __device__ int64_t upto(int n, const RowsArgs& a) const {  // of the first n blocks
    const int64_t m = min(n, linear);
    return m * (first + kRowsCost) + m * (m + 1) / 2 * a.qpb + (int64_t)(n - m) * ((int64_t)most + kRowsCost);
  }
};

__device__ inline int64_t lane_of(int64_t v, int l) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 |
                   (uint32_t)__builtin_amdgcn_readlane((int)v, l));
}

// The same in all lanes, and known to be.
__device__ inline int same(int v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ inline int64_t same(int64_t v) {
  return (int64_t)((uint64_t)(uint32_t)same((int)(v >> 32)) << 32 | (uint32_t)same((int)v));
}

// The same number, as one that the compiler knows nothing of: what follows from it is worked out here.
__device__ __forceinline__ int anew(int v) {
  asm volatile("" : "+v"(v));
  return v;
}

// Where the count stands: a block, and how far into it.
struct RowsAt {
  int s, hs, qb;     // sequence, K/V head and part of its group, block of queries
  int64_t at;        // into the block
};

// Two numbers, and products of tiles, in bf16 or fp16.
template <bool F16>
__device__ __forceinline__ uint32_t pack_two(float lo, float hi) {
  if constexpr (!F16) return pack_bf16(lo, hi);
  typedef _Float16 f16v2 __attribute__((ext_vector_type(2)));
  const f16v2 v = __builtin_convertvector(f32v2{lo, hi}, f16v2);  // round to nearest even
  uint32_t u;
  __builtin_memcpy(&u, &v, 4);
  return u;
}
template <bool F16>
__device__ __forceinline__ float low_of(uint32_t w) {
  if constexpr (!F16) return __uint_as_float(w << 16);
  const uint16_t h = (uint16_t)w;
  _Float16 v;
  __builtin_memcpy(&v, &h, 2);
  return (float)v;
}
template <bool F16>
__device__ __forceinline__ float high_of(uint32_t w) {
  return F16 ? low_of<F16>(w >> 16) : __uint_as_float(w & 0xffff0000u);
}
template <bool F16>
__device__ __forceinline__ f16x mma32(const u32x4& a, const u32x4& b, f16x c) {
  if constexpr (!F16) return mma32_bf16(a, b, c);
  typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
  f16x8 av, bv;
  __builtin_memcpy(&av, &a, 16);
  __builtin_memcpy(&bv, &b, 16);
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(av, bv, c, 0, 0, 0);
}
// The power of two that numbers of at most `top` are divided by so that it lies in [2^lo, 2^hi): 0 where it does, else
// one that brings it to the upper bound.
__device__ __forceinline__ int power_of(float top, int lo, int hi) {
  const int e = (int)(__float_as_uint(top) >> 23) - 127;
  return top == 0.f || e == 128 || (e >= lo && e < hi) ? 0 : e - (hi - 1);
}
// Keys and values in fp16 are 2^6 of themselves, for more small ones: those of a token reach from 2^-2 to 2^8 (24 times a
// scale of 4 bits is then below 2^16).  Values are in units of 2^-4 by themselves, as they are the smaller ones in
// models: from 2^-6 to 2^4; where the first two tiles' largest one is near a bound of that or past it, of one that it is the
// middle of.  On 16384 tokens in 8 bits, 64 heads on 8, values of 1/16 root mean square (with units of 1 most of their tokens are
// below 1/4): 2048 new ones 2991 us with units of 1 and 1086 so, 128 231 and 126.  2048 with values of 8, where the numbers
// that are made before do not fit, 1490, and 1131 with values of 4.
constexpr int kRowsBoost = 6, kRowsLo = -2, kRowsHi = 8, kRowsUnit = -4;
constexpr int kRowsZero = -512;        // the power of a token whose values are all 0: below any other's
constexpr uint32_t kRowsDead = ~0u;    // scales of a key that no query of a block sees (kv_encode stores no such NaN)
constexpr int kRowsFold = 60;          // sums lie within 2^+-60 of what they are relative to, or have a power of their own

template <int FMT, int HD>
struct RowsGeo {
  static constexpr bool QUANT = FMT == DUO_KV_I8 || FMT == DUO_KV_I4;
  static constexpr int KB = 64, CH = HD / 8, TILE = KB * CH;  // keys of a tile, 16-byte chunks per row, of a tile
  static constexpr int RB = KvFmt<FMT>::row(HD);
  static constexpr int NL = QUANT ? 1 + (16 * RB > 1024) : 16 * RB / 1024;  // loads of 16 rows
  static constexpr int STAGE = QUANT ? NL * 1024 : 0;                       // of a wave and operand
  static constexpr int LDS = 4 * TILE * 16 + 8 * STAGE;
};

template <int FMT, int HD>
__global__ __launch_bounds__(256, 2) void rows_kernel(RowsArgs a) {
  using G = RowsGeo<FMT, HD>;
  constexpr int KB = G::KB, CH = G::CH, TILE = G::TILE, RB = G::RB, NL = G::NL, QB = kRowsQB;
  constexpr bool MADE = FMT == kKvMade, F16 = G::QUANT || MADE;
  constexpr int KS = HD / 16, DB = HD / 32;  // MFMA steps over head_dim, 32-wide blocks of the output row
  constexpr int RPL = 64 / CH;               // rows of bf16 per wave-wide access
  extern __shared__ __attribute__((aligned(16))) uint8_t lsm[];
  u32x4* const sm = (u32x4*)lsm;  // [buffer][K, V][tile]
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int nhs = a.kv.heads * a.nsub;

  if (a.flags) {
    bool some = false;
#pragma unroll 4
    for (int i = lane * 16; i < a.nflags; i += 1024) {
      const u32x4 v = *(const u32x4*)(a.flags + i);
      some |= (v[0] | v[1] | v[2] | v[3]) != 0;
    }
    // numbers that do not fit: the rows that were made are left, and their sequences done from the codes
    a.most = (__any(some) != 0) == MADE ? (MADE ? 0 : a.over) : INT64_MAX;
  }
  // ---- the count, and this workgroup's share of it
  RowsSeq mine(a, a.per == 1 ? lane : a.nseq);
  int64_t upto = 0;
  if (a.per == 1)
    upto = mine.upto(mine.nb, a) * nhs;
  else
    for (int i = 0; i < a.per; ++i) {
      const RowsSeq q(a, (int)min((int64_t)lane * a.per + i, (int64_t)a.nseq));
      upto += q.upto(q.nb, a) * nhs;
    }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t v = __shfl_up(upto, o);
    upto += lane >= o ? v : 0;
  }
  const int64_t total = lane_of(upto, 63);
  const uint64_t made = __ballot(mine.nb + mine.dealt > 0);  // MADE: which sequences the rows are of
  const int shares = (int)min((int64_t)gridDim.x, (total + kRowsMin - 1) / kRowsMin);
  const int64_t size = same(shares ? (int64_t)rows_div(total, shares) : 0);
  const int more = (int)(total - size * shares);
  auto begin = [&](int i) { return i * size + min(i, more); };
  auto share_of = [&](int64_t u) {
    const int64_t cut = more * (size + 1);
    return u < cut ? (int)rows_div(u, size + 1) : more + (int)rows_div(u - cut, size);
  };
  // workgroups (a multiple of eight) go round-robin over the XCDs, neighbouring shares to one
  const int share = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
  if (tid == 0) a.tasks[share].parts = 0;
  auto load_seq = [&](int s) {
    RowsSeq q(a, s);
    q.dealt = same(q.dealt);
    q.q0 = same(q.q0), q.lq = same(q.lq), q.len = same(q.len), q.nb = same(q.nb);
    q.first = same(q.first), q.most = same(q.most), q.linear = same(q.linear);
    return q;
  };
  auto seq_of = [&](int s) {
    if (a.per > 1) return load_seq(s);
    RowsSeq q = mine;
    q.dealt = __builtin_amdgcn_readlane(mine.dealt, s);
    q.q0 = __builtin_amdgcn_readlane(mine.q0, s), q.lq = __builtin_amdgcn_readlane(mine.lq, s);
    q.len = __builtin_amdgcn_readlane(mine.len, s), q.nb = __builtin_amdgcn_readlane(mine.nb, s);
    q.first = __builtin_amdgcn_readlane(mine.first, s), q.most = __builtin_amdgcn_readlane(mine.most, s);
    q.linear = __builtin_amdgcn_readlane(mine.linear, s);
    return q;
  };
  auto locate = [&](int64_t u) {  // u < total
    const int bucket = __ffsll((unsigned long long)__ballot(upto > u)) - 1;
    if (bucket) u -= lane_of(upto, bucket - 1);
    RowsAt p;
    for (p.s = bucket * a.per;; ++p.s) {
      const RowsSeq q = seq_of(p.s);
      const int64_t each = q.upto(q.nb, a);
      if (u >= each * nhs) {
        u -= each * nhs;
        continue;
      }
      p.hs = same((int)rows_div(u, each));
      u = same(u - p.hs * each);
      // the block: by the root of the count (or its even part), put right by whole numbers
      const double b = (double)q.first + kRowsCost + 0.5 * a.qpb, v = (double)u;
      double x = (sqrt(b * b + 2.0 * a.qpb * v) - b) / a.qpb;
      const int64_t even = q.upto(q.linear, a);
      if (u >= even) x = (double)q.linear + (double)(u - even) / ((double)q.most + kRowsCost);
      int lo = same(min(max((int)x, 0), q.nb - 1));
      while (lo > 0 && same((int)(q.upto(lo, a) > u))) --lo;
      while (lo < q.nb - 1 && same((int)(q.upto(lo + 1, a) <= u))) ++lo;
      p.qb = lo;
      p.at = same(u - q.upto(lo, a));
      return p;
    }
  };
  auto near = [&](int c) { return (int)min((int64_t)min(kRowsSnap, c / 2), size / 2); };
  // a place in a block moved to the block's edge that is near, if any
  auto snap = [&](int64_t u, const RowsAt& p, int c) {
    return same(p.at <= near(c) ? u - p.at : c - p.at <= near(c) ? u - p.at + c : u);
  };
  auto advance = [&](RowsAt& p, RowsSeq& q, auto load) {  // to the block behind this one, which there is
    p.at = 0;
    if (++p.qb < q.nb) return;
    p.qb = 0;
    if (++p.hs < nhs) return;
    p.hs = 0;
    do
      q = load(++p.s);
    while (q.nb == 0);
  };
  // the share [u, u1), and where it begins
  int64_t u = 0, u1 = 0;
  RowsAt p = {}, start = {};
  if (share < shares) {
    u = same(begin(share)), u1 = same(begin(share + 1));
    if (u1 < total) {
      const RowsAt e = locate(u1);
      u1 = snap(u1, e, seq_of(e.s).cost(e.qb, a));
    }
    start = locate(u);
    RowsSeq q = seq_of(start.s);
    const int c = q.cost(start.qb, a);
    const int64_t to = snap(u, start, c);
    start.at = same(start.at + to - u);
    u = to;
    if (u < u1 && start.at == c) advance(start, q, seq_of);
  }
  // what is dealt out comes first: from sequence s on, the next that has some, in rounds
  int s_next = -1, round = 0, rounds = 0;
  RowsSeq q{};
  auto dealt_seq = [&]() {
    for (int s = s_next + 1; s < a.nseq; s += 64) {
      const RowsSeq x(a, s + lane);
      const uint64_t some = __ballot(x.dealt > 0);
      if (some) {
        s_next = s + __ffsll((unsigned long long)some) - 1;
        q = load_seq(s_next);
        round = 0, rounds = q.dealt / a.deal;
        return;
      }
    }
    rounds = 0;
  };
  if (a.deal) dealt_seq();
  bool dealing = rounds > 0;
  if (!dealing && u < u1) p = start, q = load_seq(p.s);

  while (dealing || u < u1) {
    if (dealing) {
      // a round takes a.deal blocks of every head, the last ones first and every other round from its short end
      const int head = (int)blockIdx.x % nhs, j = (int)blockIdx.x / nhs;
      p.s = s_next, p.hs = same(head), p.at = 0;
      p.qb = same(q.nb + q.dealt - 1 - (round * a.deal + (round & 1 ? a.deal - 1 - j : j)));
    }
    const int cost = dealing ? kRowsAll : q.cost(p.qb, a);  // all of a block that is dealt out
    const int64_t block = u - p.at;  // where it begins in the count
    const int from_at = same((int)p.at), to_at = same(dealing ? cost : (int)min((int64_t)cost, u1 - block));
    const int kvh = same(p.hs / a.nsub), sub = same(p.hs - kvh * a.nsub);
    const int heads = min(a.hg, a.group - sub * a.hg), head0 = kvh * a.group + sub * a.hg;
    const int qi0 = same(p.qb * a.qpb), rows = same(min(a.qpb, q.lq - qi0) * a.hg);
    const int len = same(q.len), pos0 = same(len - q.lq + qi0);  // position of the block's first query
    const int32_t* const pages = a.table + same((int64_t)p.s * a.ldt);
    const int seq_q0 = same(q.q0);
    const uint32_t made0 = MADE ? (uint32_t)same((int)__popcll(made & (((uint64_t)1 << p.s) - 1)) * a.made_tiles) : 0u;
    // on to the next block
    if (dealing) {
      if (++round == rounds) {
        dealt_seq();
        dealing = rounds > 0;
        if (!dealing && u < u1) p = start, q = load_seq(p.s);
      }
    } else {
      u = same(block + to_at);
      if (u < u1) advance(p, q, load_seq);
    }
    // the block's tiles: `sinks` first ones, then those from `from` on; here: [t0, t0 + n)
    const int pos_end = same(pos0 + by(rows - 1, a));  // of its last query
    const int first = same(a.window ? max(pos0 - a.window + 1, 0) : 0);
    const int sinks = same((min(a.sinks, first) + KB - 1) / KB), from = same(max(first / KB, sinks));
    const int tiles = same(pos_end < 0 ? 0 : sinks + (pos_end + KB) / KB - from);
    auto tile_at = [&](int x) { return min(max((x - kRowsCost + KB - 1) / KB, 0), tiles); };
    const int t0 = same(tile_at(from_at)), n = same(tile_at(to_at) - t0);
    const bool whole = n == tiles;
    if (n == 0 && !(tiles == 0 && from_at == 0)) continue;
    auto place = [&](int t) { return t < sinks ? t : t - sinks + from; };  // t: of all the block's tiles
    lds_barrier();  // every wave is done with the block before
    // the lane's number anew for every block: what is worked out from it would be kept, for all parts of
    // this loop at once, in more registers than there are
    const int ln = anew(lane), half = ln >> 5;
    // chunk c of key r sits at position kswz(r, c) (vswz) of its row in a tile
    auto kswz = [](int key, int c) { return CH == 16 ? c ^ (key & 15) : c ^ ((key >> 1) & 7); };
    auto vswz = [](int key, int c) { return CH == 16 ? c ^ (4 * (key & 3)) : c ^ (4 * ((key >> 1) & 1)); };
    // transposing read of 16 keys x 32 channels: lane i of each 16 addresses key i / 4, 4 values at 4 (i % 4)
    auto v_at = [&](int x, int d) {
      const int tj = (x & 15) >> 2;
      return (4 * (x >> 5) + tj) * HD * 2 + vswz(tj, 4 * d + 2 * ((x >> 4) & 1)) * 16 + (x & 3) * 8;
    };
    typedef __attribute__((address_space(3))) s16v4 lds4;
    auto read_v = [&](const uint8_t* sV, int t, int d, int x) {
      const int at = v_at(x, d);
      const s16v4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(sV + at + (16 * t) * HD * 2));
      const s16v4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(sV + at + (16 * t + 8) * HD * 2));
      u32x4 v;
      __builtin_memcpy(&v, &v0, 8);
      __builtin_memcpy((char*)&v + 8, &v1, 8);
      return v;
    };
    auto k_rows = [&](int u) { return sm + ((u >> 1 & 1) * 2) * TILE + (u & 1) * 32 * CH; };
    auto v_rows = [&](int u) { return (const uint8_t*)(sm + ((u >> 1 & 1) * 2 + 1) * TILE) + (u & 1) * 32 * HD * 2; };
    auto read_k = [&](const u32x4* sK, int c, int x) { return sK[(x & 31) * CH + kswz(x & 31, 2 * c + (x >> 5))]; };

    // ---- pages
    const int last_page = (len - 1) >> a.kv.shift, page_mask = (1 << a.kv.shift) - 1;
    const uint8_t* const block0 = a.kv.data + kvh * a.kv.block;
    const uint32_t page_bytes = (uint32_t)(a.kv.heads * a.kv.block);
    int win = n ? (place(t0) * KB >> a.kv.shift) & ~3 : 0;
    auto ids = [&](int pg) { return pages[min(pg + lane, last_page)]; };
    auto page = [&](int v) { return (uint32_t)((uint32_t)v < (uint32_t)a.kv.pages ? v : 0); };  // at most 2^31 - 1 pages
    int pid = 0, nid = 0;
    bool lost = false;  // some query sees a token in a page outside the cache
    if (n && !MADE) {  // (rows made of pages that are not there are NaN)
      pid = ids(win);
      nid = ids(win + 64);
      const int p1 = min(place(t0 + n - 1) * KB + KB - 1, pos_end) >> a.kv.shift;
      for (int pg = place(t0) * KB >> a.kv.shift; pg <= p1;) {
        int v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = pages[min(pg + 64 * j + lane, last_page)];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int i = pg + 64 * j + lane, k = i << a.kv.shift;
          lost |= i <= p1 && (v[j] < 0 || v[j] >= a.kv.pages) && (k + page_mask >= first || k < a.sinks);
        }
        pg += 256;
        if (pg << a.kv.shift >= a.sinks) pg = max(pg, first >> a.kv.shift);
      }
      lost = __any(lost);
    }
    // this wave's 16 keys of a tile (as far as there are any): their page's block, where they begin in it, and
    // the last that there is
    struct Run {
      const uint8_t* block;
      int in, left;
    };
    auto run_at = [&](int t) {  // tiles in order
      const int key = min(place(t) * KB + 16 * wave, (len - 1) & ~15), pg = key >> a.kv.shift;
      if constexpr (MADE) return Run{block0 + (uint64_t)(made0 + (uint32_t)pg) * page_bytes, key & page_mask, len - 1 - key};
      if (pg >= win + 64) {
        if (pg >= win + 128) {  // the first tile behind the sinks
          win = (pg & ~3) - 64;
          nid = ids(win + 64);
        }
        pid = nid;
        win += 64;
        nid = ids(win + 64);
      }
      const uint32_t id = page(__builtin_amdgcn_readlane(pid, pg - win));
      return Run{block0 + (uint64_t)id * page_bytes, key & page_mask, len - 1 - key};
    };
    // where a lane's 16 bytes come from; the same for all loads of V's 16 rows, and of codes (16 rows of 32
    // bytes fill half a load: the others again)
    uint32_t k_off[NL], v_off[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int r = ln / CH, c = ln % CH;
      k_off[i] = G::QUANT ? ln * 16 % (16 * RB) : r * RB + 16 * kswz(i * RPL + r, c);
      v_off[i] = G::QUANT ? ln * 16 % (16 * RB) : r * RB + 16 * vswz(r, c);
    }
    auto issue = [&](const Run& run, auto which_c, const void* to) __attribute__((always_inline)) {
      constexpr int which = decltype(which_c)::value;
      const uint32_t lds = __builtin_amdgcn_readfirstlane(lds_addr(to));
      const uint8_t* const at = run.block + (kv_rows_at<FMT, HD>(which, a.kv.shift) + run.in * RB);
      if (run.left >= 15) {
        if constexpr (NL > 1)
          dma16_run<NL>(at, which ? v_off : k_off, lds);
        else
          dma16(at, which ? v_off[0] : k_off[0], lds);
        return;
      }
      const int x = anew(lane);  // rows past the last as the last
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        if constexpr (!G::QUANT) {
          const int r = i * RPL + x / CH, c = x % CH;
          dma16(at, min(r, run.left) * RB + 16 * (which ? vswz(r, c) : kswz(r, c)), lds + i * 1024);
        } else {
          const int e = (i * 1024 + x * 16) % (16 * RB);
          dma16(at, min(e / RB, run.left) * RB + e % RB, lds + i * 1024);
        }
      }
    };
    constexpr std::integral_constant<int, 0> kK{};
    constexpr std::integral_constant<int, 1> kV{};
    // ---- 8 and 4 bits
    uint8_t* const stage = lsm + 4 * TILE * 16 + wave * 2 * G::STAGE;  // codes of K, then of V
    // A thread makes numbers of one key of its wave's run and HD / 4 channels, whose scale it loads; a lane also
    // looks at all scales of one key of the tile, for the powers.
    struct Scales {
      uint32_t w[HD / 64];
    };
    const uint32_t v_scales = (uint32_t)KvFmt<FMT>::scales(HD) << a.kv.shift;  // from K's on
    auto scale_of = [&](const Run& run, uint16_t* k, uint16_t* v) {
      const int x = anew(lane);
      const uint8_t* const s = run.block + (kv_scales_at<FMT, HD>(0, a.kv.shift) + run.in * KvFmt<FMT>::scales(HD));
      const uint32_t off = (uint32_t)(min(x >> 2, run.left) * KvFmt<FMT>::scales(HD) + (HD == 128 ? x & 3 : x >> 1 & 1) * 2);
      *k = *(const uint16_t*)(s + off);
      *v = *(const uint16_t*)(s + v_scales + off);
    };
    auto scales_of = [&](const Run& run, int t, Scales* k, Scales* v) {  // after run_at(t)
      const int x = anew(lane), key = min(place(t) * KB + (a.kv.shift < 6 ? x & 48 : 0), (len - 1) & ~15);
      constexpr int SB = KvFmt<FMT>::scales(HD);
      const uint8_t* block = run.block;
      if (a.kv.shift < 6) block = block0 + (uint64_t)page(__shfl(pid, (key >> a.kv.shift) - win)) * page_bytes;
      const uint8_t* const s = block + (kv_scales_at<FMT, HD>(0, a.kv.shift) + (key & page_mask) * SB);
      const uint32_t off = (uint32_t)(min(a.kv.shift < 6 ? x & 15 : x, len - 1 - key) * SB);
      auto load = [&](const uint8_t* at, Scales* r) {
        if constexpr (HD == 128) {
          const uint2 w = *(const uint2*)(at + off);
          r->w[0] = w.x, r->w[HD / 64 - 1] = w.y;
        } else {
          r->w[0] = *(const uint32_t*)(at + off);
        }
      };
      load(s, k);
      load(s + v_scales, v);
      // keys that no query of the block sees have no say in the powers
      const int k0 = place(t) * KB;
      if (lost || k0 + KB - 1 > pos_end || (k0 < first && k0 + KB > a.sinks)) {
        const int seen = k0 + x;
        const int id = __shfl(pid, (min(seen, len - 1) >> a.kv.shift) - win);
        // (without a branch of its own: lanes that part here made the compiler take pages' addresses for theirs)
        const uint32_t dead = (seen > pos_end) | ((seen < first) & (seen >= a.sinks)) | (id < 0) | (id >= a.kv.pages) ? kRowsDead : 0u;
#pragma unroll
        for (int i = 0; i < HD / 64; ++i) k->w[i] |= dead, v->w[i] |= dead;
      }
    };
    // the largest number that the key's codes can stand for (a scale that is NaN aside)
    auto most_of = [&](const Scales& s) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < HD / 64; ++i) {
        const uint32_t lo = s.w[i] & 0xffffu, hi = s.w[i] >> 16;
        m = max(m, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
      }
      if constexpr (G::QUANT) return __uint_as_float(m << 16) * KvFmt<FMT>::most;
      return 0.f;
    };
    auto k_power = [&](const Scales& s) { return power_of(most_of(s), kRowsLo, kRowsHi); };
    // power of two that the outputs are in units of: another one where the first two tiles' values ask for it (the first one
    // may hold sinks alone, whose values are often small)
    int e_ref = kRowsUnit;
    // Small values go to the lower bound only: what a probability loses to its value's power it lacks in fp16, and
    // beside values just above the bound ones just below it would lose 2^10 at once.
    auto v_power = [&](const Scales& s) {
      const float most = most_of(s);
      const int e = (int)(__float_as_uint(most) >> 23) - 127 - e_ref;
      if (most == 0.f) return s.w[0] == kRowsDead ? 0 : kRowsZero;
      return e < kRowsLo ? e - kRowsLo : e < kRowsHi ? 0 : e - (kRowsHi - 1);
    };
    // does some key's largest scale mean a power, as far as one look can tell (never no for yes)?
    auto some_power = [&](const Scales& k, const Scales& v) {
      typedef unsigned short u16v2 __attribute__((ext_vector_type(2)));
      auto most = [](const Scales& s) {
        u16v2 m;
        __builtin_memcpy(&m, &s.w[0], 4);
        if constexpr (HD == 128) {
          u16v2 o;
          __builtin_memcpy(&o, &s.w[HD / 64 - 1], 4);
          m = __builtin_elementwise_max(m, o);
        }
        return (uint32_t)(m[0] > m[1] ? m[0] : m[1]);
      };
      if constexpr (G::QUANT) {
        // scales whose code of most lies within the bounds, bf16 numbers as whole ones
        constexpr uint32_t lo = ((127u + kRowsLo) << 7) - (KvFmt<FMT>::most == 127 ? 6 << 7 : 2 << 7);
        constexpr uint32_t hi = ((127u + kRowsHi) << 7) - (KvFmt<FMT>::most == 127 ? 7 << 7 : 3 << 7);
        return __any(most(k) - lo >= hi - lo || most(v) - (lo + kRowsUnit * 128) >= hi - lo) != 0;
      }
      return false;
    };
    // power: what the lane's key is divided by, where odd (values' units aside)
    auto convert = [&](const uint8_t* codes, uint16_t scale, bool odd, int power, u32x4* tile, bool is_v) __attribute__((always_inline)) {
      if constexpr (G::QUANT) {
        constexpr int NC = HD / 4;  // channels
        typedef _Float16 f16v2 __attribute__((ext_vector_type(2)));
        const int x = anew(lane), ckey = x >> 2, cpart = x & 3, key = 16 * wave + ckey;
        int up = is_v ? kRowsBoost - e_ref : kRowsBoost;
        if (odd) up -= __shfl(power, key);
        const _Float16 s1 = (_Float16)ldexpf(bf16_bits_to_f32(scale), up);
        const f16v2 s = {s1, s1};
        const uint8_t* const at = codes + ckey * RB + cpart * (RB / 4);
        uint32_t w[RB / 16];
#pragma unroll
        for (int i = 0; i < RB / 16; i += 2) {
          const uint2 two = *(const uint2*)(at + 4 * i);
          w[i] = two.x, w[i + 1] = two.y;
        }
        auto as_h = [](uint32_t u) {
          f16v2 h;
          __builtin_memcpy(&h, &u, 4);
          return h;
        };
#pragma unroll
        for (int j = 0; j < NC / 8; ++j) {
          u32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            f16v2 h;
            if constexpr (FMT == DUO_KV_I8) {
              // a byte b below 0x64 is the number 1024 + b
              const f16v2 excess = {(_Float16)-1152.f, (_Float16)-1152.f};
              h = (as_h(__builtin_amdgcn_perm(0x64646464u, w[2 * j + (e >> 1)], e & 1 ? 0x04030402u : 0x04010400u)) + excess) * s;
            } else {
              // a nibble n in bits 6 to 9 of 0x4c00 is 16 + n, and 24 s is exact; channels e and e + 4 together
              const uint32_t n = e == 0 ? w[j] << 6 : e == 1 ? w[j] << 2 : e == 2 ? w[j] >> 2 : w[j] >> 6;
              h = __builtin_elementwise_fma(as_h((n & 0x03c003c0u) | 0x4c004c00u), s, s * (_Float16)-24.f);
            }
            uint32_t two;
            __builtin_memcpy(&two, &h, 4);
            v[e] = two;
          }
          const int c = cpart * (NC / 8) + j;
          tile[key * CH + (is_v ? vswz(key, c) : kswz(key, c))] = v;
        }
      }
    };
    // Of the next codes to become numbers, and of the V after: scales.
    uint16_t ks = 0, vs = 0, vs1 = 0;
    Scales kall = {}, vall = {};
    // powers of the lane's key and value in this tile, the next and the one after; are there any?
    int kp = 0, kp1 = 0, kp2 = 0, vp = 0, vp1 = 0, vp2 = 0;
    bool odd = false, odd1 = false, odd2 = false, calm = true;
    int odd_l = 0;  // has some row's sum a power (which it gets in a tile that is odd)?
    auto powers = [&](int* k, int* v) {
      bool some = e_ref != kRowsUnit || some_power(kall, vall);
      if (some) {
        *k = k_power(kall), *v = v_power(vall);
        some = __any((*k | *v) != 0);
      } else {
        *k = *v = 0;
      }
      return some;
    };
    auto next = [&]() __attribute__((always_inline)) {  // on to the next tile
      if constexpr (G::QUANT) {
        kp = kp1, kp1 = kp2, vp = vp1, vp1 = vp2;
        odd = odd1, odd1 = odd2;
        calm = !(odd | odd1);
      }
    };
    auto tile_of = [&](int i, int which) { return sm + ((i & 1) * 2 + which) * TILE; };  // i: of the tiles here
    auto mine_of = [&](int i, int which) { return tile_of(i, which) + wave * 16 * CH; };

    // ---- the first tiles and the queries are on their way together
    const int row0 = 32 * wave;
    struct Row {
      int qi, head;
    };
    auto row_of = [&](int x) {
      const int row = min(row0 + (x & 31), rows - 1), qi = by(row, a);
      return Row{qi, row - qi * a.hg};
    };
    const int pos_lo = pos0 + by(min(row0, rows - 1), a), pos_hi = pos0 + by(min(row0 + 31, rows - 1), a);  // of this wave
    Run run_v = {};  // of the tile whose V comes next
    if (n) {
      const Run run0 = run_at(t0);
      if constexpr (!G::QUANT) {
        issue(run0, kK, mine_of(0, 0));
        if (n > 1) {
          run_v = run_at(t0 + 1);
          issue(run_v, kK, mine_of(1, 0));
        }
        issue(run0, kV, mine_of(0, 1));
      } else {
        uint8_t* const k1 = (uint8_t*)tile_of(1, 1) + wave * G::STAGE;  // the second K's codes: V's second tile comes later
        issue(run0, kK, stage);
        issue(run0, kV, stage + G::STAGE);
        scale_of(run0, &ks, &vs);
        scales_of(run0, t0, &kall, &vall);
        Scales kall1 = {}, vall1 = {};
        uint16_t ks1 = 0;
        if (n > 1) {
          run_v = run_at(t0 + 1);
          issue(run_v, kK, k1);
          scale_of(run_v, &ks1, &vs1);
          scales_of(run_v, t0 + 1, &kall1, &vall1);
        }
        wait_vm<0>();
        asm volatile("" ::: "memory");
        float m = fmaxf(most_of(vall), most_of(vall1));
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
        const int e_most = same((int)(__float_as_uint(m) >> 23)) - 127, middle = (kRowsLo + kRowsHi) / 2;
        // near a bound, or past it: the middle, so that the other tokens are not on both sides of it
        if (same((int)(m > 0.f)) && (e_most < kRowsLo + kRowsUnit + 2 || e_most >= kRowsHi + kRowsUnit - 2)) e_ref = e_most - middle;
        odd = powers(&kp, &vp);
        convert(stage, ks, odd, kp, tile_of(0, 0), false);
        convert(stage + G::STAGE, vs, odd, vp, tile_of(0, 1), true);
        if (n > 1) {
          kall = kall1, vall = vall1;
          odd1 = powers(&kp1, &vp1);
          convert(k1, ks1, odd1, kp1, tile_of(1, 0), false);
        }
        calm = !(odd | odd1);
        wait_lds<0>();
        vs = vs1;
        const Run run1 = run_v;
        if (n > 2) {
          run_v = run_at(t0 + 2);
          issue(run_v, kK, stage);
          scale_of(run_v, &ks, &vs1);
          scales_of(run_v, t0 + 2, &kall, &vall);
        }
        if (n > 1) issue(run1, kV, stage + G::STAGE);
      }
    }
    u32x4 qa[KS];
    {
      const Row w = row_of(ln);
      const uint16_t* const at = a.Q + (int64_t)(seq_q0 + qi0 + w.qi) * a.ldq + (int64_t)(head0 + min(w.head, heads - 1)) * HD;
#pragma unroll
      for (int c = 0; c < KS; ++c) qa[c] = *(const u32x4*)(at + 8 * (2 * c + half));
#pragma unroll
      for (int c = 0; c < KS; ++c) {
        asm volatile("" : "+v"(qa[c]));
#pragma unroll
        for (int j = 0; j < 4; ++j) qa[c][j] ^= a.flip;
      }
    }
    int q_power = 0;  // of the lane's row
    if constexpr (F16) {
      uint32_t top = 0;
#pragma unroll
      for (int c = 0; c < KS; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t w = qa[c][j] & 0x7fff7fffu;
          top = max(top, max(w & 0xffffu, w >> 16));
        }
      const auto x = __builtin_amdgcn_permlane32_swap(top, top, false, false);
      q_power = power_of(__uint_as_float(max(x[0], x[1]) << 16), -3, 15);
#pragma unroll
      for (int c = 0; c < KS; ++c)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          qa[c][j] = pack_two<F16>(ldexpf(__uint_as_float(qa[c][j] << 16), -q_power), ldexpf(__uint_as_float(qa[c][j] & 0xffff0000u), -q_power));
      if constexpr (FMT == DUO_KV_I4)  // channels e and e + 4 together, as the keys have them
#pragma unroll
        for (int c = 0; c < KS; ++c) {
          const u32x4 v = qa[c];
          qa[c] = u32x4{(v[0] & 0xffffu) | v[2] << 16, v[0] >> 16 | (v[2] & 0xffff0000u), (v[1] & 0xffffu) | v[3] << 16,
                        v[1] >> 16 | (v[3] & 0xffff0000u)};
        }
    }
    const bool odd_q = __any(q_power != 0);
    float m = -INFINITY, mc = -INFINITY, l = 0.f;  // reference, times cexp; sum of this half's keys
    int l_power = 0;  // (8 and 4 bits) the sum is l 2^l_power
    f16x o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    // Steps of 32 keys, two per tile, counted from t0.  This wave: steps up to nu have keys that its
    // queries see, those in [f0, f1) are seen whole by all of them.
    const int shift = 2 * (sinks - from - t0);  // of a step behind the sinks, from its keys' number / 32
    const int nu = row0 >= rows || pos_hi < 0 ? 0 : min(max((pos_hi >> 5) + 1 + shift, 0), 2 * n);
    const int f0 = lost ? 2 * n : !a.window ? 0 : max((max(pos_hi - a.window + 1, 0) + 31) / 32, 2 * from) + shift;
    const int f1 = lost ? 2 * n : max(pos_lo + 1, 0) / 32 + shift;
    auto first_key = [&](int u) { return place(t0 + (u >> 1)) * KB + (u & 1) * 32; };
    const int fast_end = odd_q ? 0 : same(min(nu - 4, f1 - 3));  // of two tiles' first step
    const uint32_t nf = (uint32_t)same(max(f1 - f0, 0));
    auto masked = [&](int u) { return (uint32_t)(u - f0) >= nf; };
    // of the query at position pos
    const int back = a.window ? a.window : kRowsBack;
    auto sees = [&](int pos, int key) { return key <= pos && (key > pos - back || key < a.sinks); };

    f16x sa, sb;  // scores of an even and of an odd step
    u32x4 pf[2];  // probabilities of a step
    auto score = [&](int u, f16x& sc) __attribute__((always_inline)) {
      const int x = anew(lane);
#pragma unroll
      for (int r = 0; r < 16; ++r) sc[r] = 0.f;
#pragma unroll
      for (int c = 0; c < KS; ++c) sc = mma32<F16>(read_k(k_rows(u), c, x), qa[c], sc);
    };
    // a new reference where the step's scores leave the old one's range: the factor of what is
    // relative to the old one (1 elsewhere), and whether any lane has one
    // units: the scores' in the exponent of two (a.cexp, or 1 where they are that already)
    auto refer = [&](const f16x& sc, float* f, float units) __attribute__((always_inline)) {
      float mt = sc[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) mt = fmaxf(mt, sc[r]);
      const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
      mt = fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
      if constexpr (F16) {
        mt *= units;
        const bool up = mt > mc + 8.f;
        if (!__any(up)) return false;
        *f = up ? mc == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - mt) : 1.f;
        mc = up ? mt : mc;
        l *= *f;
        return true;
      }
      const bool up = mt > m && !(mt * a.cexp <= mc + 8.f);
      if (!__any(up)) return false;
      const float mcn = up ? mt * a.cexp : mc;
      *f = up ? m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - mcn) : 1.f;
      m = up ? mt : m;
      mc = mcn;
      l *= *f;
      return true;
    };
    auto written = [&]() __attribute__((always_inline)) {  // the last products have been
#pragma unroll
      for (int d = 0; d < DB; ++d) asm volatile("s_nop 15" : "+v"(o[d]));
    };
    auto scale_o = [&](float f) __attribute__((always_inline)) {
      written();
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= f;
    };
    // What probabilities are relative to: in fp16 the reference's is 2^6, as small ones have fewer bits there
    auto base_of = [&]() { return F16 ? mc - 6.f : mc; };
    auto probabilities = [&](const f16x& sc, u32x4 (&p)[2], float units) __attribute__((always_inline)) {
      const float base = (F16 ? mc : m) == -INFINITY ? 0.f : base_of();
      float sum = 0.f;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(sc[8 * t + 2 * j], units, -base));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(sc[8 * t + 2 * j + 1], units, -base));
          sum += p0 + p1;
          p[t][j] = pack_two<F16>(p0, p1);
        }
      return sum;
    };
    // O += V^T P^T of step u
    auto add = [&](int u) __attribute__((always_inline)) {
      const uint8_t* const sV = v_rows(u);
      const int lx = anew(lane);
      u32x4 v[2][DB];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < DB; ++d) v[t][d] = read_v(sV, t, d, lx);
      if (masked(u)) {
        // some query may not see some key, and 0 times a number that is not finite would not be 0:
        // such numbers enter as zeros and are added for those who see them
        typedef unsigned short u16v2 __attribute__((ext_vector_type(2)));
        u16v2 most = {0, 0};
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t w = v[t][d][j] & 0x7fff7fffu;
              u16v2 x;
              __builtin_memcpy(&x, &w, 4);
              most = __builtin_elementwise_max(most, x);
            }
        constexpr uint32_t INF = F16 ? 0x7c00u : 0x7f80u;
        if (__any(most[0] >= INF || most[1] >= INF)) {
#pragma unroll
          for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const uint32_t w = v[t][d][j];
                v[t][d][j] = w & ~(((w & INF) == INF ? 0xffffu : 0u) | ((w >> 16 & INF) == INF ? 0xffff0000u : 0u));
              }
          written();
          const int k0 = first_key(u), pos = pos0 + row_of(lx).qi;
#pragma unroll 1
          for (int key = 0; key < 32; ++key) {
            const bool see = sees(pos, k0 + key);
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
              for (int g = 0; g < 4; ++g) {
                const uint2 w = *(const uint2*)(sV + key * HD * 2 + vswz(key, 4 * d + g) * 16 + 8 * (lx >> 5));
                const float x[4] = {low_of<F16>(w.x), high_of<F16>(w.x), low_of<F16>(w.y), high_of<F16>(w.y)};
#pragma unroll
                for (int r = 0; r < 4; ++r) o[d][4 * g + r] += see && !(fabsf(x[r]) < INFINITY) ? x[r] : 0.f;
              }
          }
        }
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = mma32<F16>(v[t][d], pf[t], o[d]);
    };
    // Step u's probabilities, the values of the step before and the scores of the next, where nothing is masked: meant to
    // be dealt out evenly, MFMAs of the one, LDS reads and vector instructions of the others.  With heads of 64 they are
    // (reads six ahead, waits for all but five); with heads of 128 the compiler leaves the groups, to keep
    // within the registers of two workgroups per CU, and each MFMA stands behind its own LDS read and a wait for
    // all of them, the exponentials in two clumps of eight: the packed kernel, from the same lines, is 5 to 7 % faster.
    auto fast = [&](auto where, f16x& sc, f16x& sn) __attribute__((always_inline)) {
      constexpr int W = decltype(where)::value;  // the step's place in two tiles, as its LDS buffers go by it
      const float base = base_of();
      const u32x4* const sK = k_rows(W + 1);
      const uint8_t* const sV = v_rows(W + 3);
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
          pn[t][j] = pack_two<F16>(p0, p1);
        }
#pragma unroll
        for (int i = 0; i < KS / 2; ++i) {
          const int c = t * (KS / 2) + i;
          sn = mma32<F16>(read_k(sK, c, ln), qa[c], sn);
          if (i < DB) o[i] = mma32<F16>(read_v(sV, t, i, ln), pf[t], o[i]);
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
      if (__any(most > (F16 ? 16384.f : 256.f) || (F16 ? mc : m) == -INFINITY)) {
        float f = 1.f;
        if (refer(sc, &f, a.cexp)) scale_o(f);
        sum = probabilities(sc, pn, a.cexp);
      }
      l += sum;
      pf[0] = pn[0];
      pf[1] = pn[1];
    };
    auto slow = [&](int u, f16x& sc, f16x& sn) __attribute__((always_inline)) {
      if (u > 0 && u <= nu) add(u - 1);
      if (u < nu) {
        if (masked(u)) {
          const int x = anew(lane), k0 = first_key(u), pos = pos0 + row_of(x).qi;
          bool gone[2] = {false, false};  // of the step's two runs of 16 keys
          if (lost)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int id = pages[min(k0 + 16 * i, len - 1) >> a.kv.shift];
              gone[i] = id < 0 || id >= a.kv.pages;
            }
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int key = k0 + 8 * (r >> 2) + 4 * (x >> 5) + (r & 3);
            sc[r] = !sees(pos, key) ? -INFINITY : gone[r >> 3] ? NAN : sc[r];
          }
        }
        float f, units = a.cexp;
        bool any_power = false;  // of a key, a value or a query
        if constexpr (F16) {
          any_power = odd_q | odd;
          if (any_power) {
            const int from_lane = (u & 1) * 32 + 4 * (anew(lane) >> 5);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const int key = from_lane + 8 * (r >> 2) + (r & 3);
              sc[r] = fmaf(ldexpf(sc[r], __shfl(kp, key) + q_power), a.cexp, (float)__shfl(vp, key));
            }
            units = 1.f;
          }
        }
        const float mc0 = mc, l0 = l;
        if (refer(sc, &f, units) && u > 0) scale_o(f);
        float sum = probabilities(sc, pf, units);
        if constexpr (G::QUANT)
          if (any_power) {
            // The sum is one of p, not of p |V|, and where values lie far apart the reference says nothing of its
            // size: it has a power of its own, and where that is small (fewer than 60 either way) none.
            constexpr int NONE = -(1 << 20);
            const int from_lane = (u & 1) * 32 + 4 * (anew(lane) >> 5);
            const float base = mc == -INFINITY ? 0.f : base_of();
            float most = -INFINITY;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              sc[r] -= (float)__shfl(vp, from_lane + 8 * (r >> 2) + (r & 3));
              most = fmaxf(most, sc[r]);
            }
            const float moved = mc0 == -INFINITY ? 0.f : fmaxf(mc0 - mc, -4096.f), whole_moved = floorf(moved);
            const int l_exp = __builtin_amdgcn_frexp_expf(l0);  // l0 2^-l_exp is in [1/2, 1)
            const int was = l0 == 0.f ? NONE : l_power + l_exp + (int)whole_moved;
            int power = most == -INFINITY ? was : max(was, (int)ceilf(fminf(fmaxf(most - base, -4096.f), 4096.f)));
            if (abs(power) <= kRowsFold || power == NONE) power = 0;
            l = l0 == 0.f ? 0.f : ldexpf(ldexpf(l0, -l_exp) * __builtin_amdgcn_exp2f(moved - whole_moved), was - power);
            l_power = power;
            odd_l = same(__any(power != 0));
            sum = 0.f;
#pragma unroll
            for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(sc[r] - base - (float)power);
          }
        l += sum;
        if (u + 1 < nu) score(u + 1, sn);
      }
    };
    // K of the next tile and V of this one are in LDS, and every wave is done with K of this one and V
    // of the one before, whose places the next ones take
    auto turn = [&](int i) __attribute__((always_inline)) {
      wait_vm<0>();
      lds_barrier();
      Run run = run_v;
      if constexpr (!G::QUANT) {
        if (i + 2 < n) {
          run = run_at(t0 + i + 2);
          issue(run, kK, mine_of(i, 0));
        }
        if (i + 1 < n) issue(run_v, kV, mine_of(i + 1, 1));
      } else {
        if (i + 2 < n) {
          odd2 = powers(&kp2, &vp2);
          convert(stage, ks, odd2, kp2, tile_of(i, 0), false);
        }
        if (i + 1 < n) convert(stage + G::STAGE, vs, odd1, vp1, tile_of(i + 1, 1), true);
        wait_lds<0>();
        vs = vs1;
        if (i + 3 < n) {
          run = run_at(t0 + i + 3);
          issue(run, kK, stage);
          scale_of(run, &ks, &vs1);
          scales_of(run, t0 + i + 3, &kall, &vall);
        }
        if (i + 2 < n) issue(run_v, kV, stage + G::STAGE);
      }
      run_v = run;
    };
    if (n) {
      if constexpr (!G::QUANT) wait_vm<0>();
      lds_barrier();
      if (nu > 0) score(0, sa);
    }
    for (int i = 0; i < n;) {
      slow(2 * i, sa, sb);
      turn(i);
      slow(2 * i + 1, sb, sa);
      next();
      if (G::QUANT && odd_l) odd = true, calm = false;
      // two tiles at a time, the odd one first, so that places in LDS are known when compiled
      for (++i; (i & 1) && 2 * i - 1 >= f0 && 2 * i < fast_end && calm; i += 2) {
        fast(std::integral_constant<int, 2>{}, sa, sb);
        turn(i);
        fast(std::integral_constant<int, 3>{}, sb, sa);
        next();
        fast(std::integral_constant<int, 0>{}, sa, sb);
        turn(i + 1);
        fast(std::integral_constant<int, 1>{}, sb, sa);
        next();
      }
    }
    if (nu > 0 && nu == 2 * n) add(nu - 1);
    written();
    // ---- out
    const int le = anew(lane);
    if constexpr (G::QUANT)
      if (__any(l_power != 0)) {  // both halves' sums with one power, the larger one of those that are not 0
        const int mine = l == 0.f ? INT32_MIN : l_power;
        const auto both = __builtin_amdgcn_permlane32_swap((uint32_t)mine, (uint32_t)mine, false, false);
        const int power = max((int)both[0], (int)both[1]);
        l = l == 0.f ? 0.f : ldexpf(l, l_power - power);
        l_power = power == INT32_MIN ? 0 : power;
      }
    const auto rl = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    float sum = __uint_as_float(rl[0]) + __uint_as_float(rl[1]);
    const int o_power = G::QUANT ? e_ref - l_power : MADE ? kRowsUnit : 0;  // of the outputs, with a sum that has none
    if (!whole) {
      float* const part = a.parts + (2 * (int64_t)share + (t0 == 0)) * rows_part(HD);
      if (t0 == 0 && tid == 0) {
        const int64_t end = block + min(kRowsCost + (tiles - 1) * KB + 1, cost - near(cost));
        a.tasks[share] = RowsTask{share_of(end - 1) - share + 1, seq_q0 + qi0, head0, heads, rows, pos0};
      }
      // the sum in [1/2, 1), its power with the reference: those of all parts are then comparable, whatever their values' sizes
      const int s_power = G::QUANT ? __builtin_amdgcn_frexp_expf(sum) : 0;
      sum = ldexpf(sum, -s_power);
      auto out = [&](float v) { return F16 ? ldexpf(v, o_power - s_power - kRowsBoost) : v; };
      if (row0 + (le & 31) < rows) {
        if (le < 32) *(float2*)(part + QB * HD + 2 * (row0 + (le & 31))) = make_float2(G::QUANT ? mc + (float)(l_power + s_power) : mc, sum);
        float* const y = part + (row0 + (le & 31)) * HD + 4 * (le >> 5);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
          for (int g = 0; g < 4; ++g)
            *(f4*)(y + 32 * d + 8 * g) = f4{out(o[d][4 * g]), out(o[d][4 * g + 1]), out(o[d][4 * g + 2]), out(o[d][4 * g + 3])};
      }
      continue;
    }
    // queries that see no key: 0; a sum of 0 (every score -inf) gives NaN
    const Row w = row_of(le);
    const float inv = pos0 + w.qi < 0 ? 0.f : 1.0f / (F16 ? ldexpf(sum, MADE ? kRowsBoost - kRowsUnit : kRowsBoost) : sum);  // as the values are
    // the power comes behind the division: outputs times it may be out of fp32's range
    auto out = [&](float v) { return G::QUANT ? ldexpf(v * inv, o_power) : v * inv; };
    uint2 y[DB][4];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        y[d][g].x = pack_bf16(out(o[d][4 * g]), out(o[d][4 * g + 1]));
        y[d][g].y = pack_bf16(out(o[d][4 * g + 2]), out(o[d][4 * g + 3]));
      }
    if (a.vec) {
      // through this wave's part of LDS, where K tiles were (every wave was done with them at the
      // last turn), so that a row is written at once, 16 bytes per lane; chunk c of row r at
      // c ^ (r % CH)
      uint8_t* const st = (uint8_t*)tile_of(wave / 2, 0) + wave % 2 * (32 * HD * 2);
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g)
          if constexpr (FMT == DUO_KV_I4) {  // channels c, c + 4, c + 1, c + 5 with c = 0 or 2
            uint16_t* const y8 = (uint16_t*)(st + (le & 31) * HD * 2 + ((4 * d + g) ^ ((le & 31) & (CH - 1))) * 16) + 2 * (le >> 5);
            y8[0] = (uint16_t)y[d][g].x, y8[4] = (uint16_t)(y[d][g].x >> 16);
            y8[1] = (uint16_t)y[d][g].y, y8[5] = (uint16_t)(y[d][g].y >> 16);
          } else {
            *(uint2*)(st + (le & 31) * HD * 2 + ((4 * d + g) ^ ((le & 31) & (CH - 1))) * 16 + 8 * (le >> 5)) = y[d][g];
          }
      wait_lds<0>();
#pragma unroll
      for (int i = 0; i < 32 / RPL; ++i) {
        const int r = i * RPL + le / CH, qr = by(min(row0 + r, rows - 1), a), h = row0 + r - qr * a.hg;
        const u32x4 v = *(const u32x4*)(st + r * HD * 2 + (le % CH ^ (r & (CH - 1))) * 16);
        if (row0 + r < rows && h < heads)
          *(u32x4*)(a.O + (int64_t)(seq_q0 + qi0 + qr) * a.ldo + (int64_t)(head0 + h) * HD + 8 * (le % CH)) = v;
      }
    } else if (row0 + (le & 31) < rows && w.head < heads) {
      uint16_t* const y0 = a.O + (int64_t)(seq_q0 + qi0 + w.qi) * a.ldo + (int64_t)(head0 + w.head) * HD + 4 * (le >> 5);
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          constexpr bool I4 = FMT == DUO_KV_I4;
          uint16_t* yp = y0 + 32 * d + 8 * g - (I4 ? 2 * (le >> 5) : 0);
          yp[0] = (uint16_t)y[d][g].x;
          yp[I4 ? 4 : 1] = (uint16_t)(y[d][g].x >> 16);
          yp[I4 ? 1 : 2] = (uint16_t)y[d][g].y;
          yp[I4 ? 5 : 3] = (uint16_t)(y[d][g].y >> 16);
        }
    }
  }
}

// Rows of sequences with more than `over` rows made of their codes, a workgroup for 64 tokens of a K/V head, as far
// as some new token sees them: pages of 64 tokens, K rows and V rows.  Rows in pages that are not there are NaN.
// A thread has eight neighbouring channels, so that a wave writes whole rows: some 17000 tokens of 8 heads of 128
// in 8 bits 22 us, bound by HBM; 34 with 32 channels a thread, whose stores are spread over 64 places each.
// flags: is there a token whose numbers do not fit as they are, or anything else against these rows?
template <int FMT, int HD>
__global__ __launch_bounds__(256) void rows_make_kernel(RowsArgs a, uint8_t* __restrict__ out, uint8_t* __restrict__ flags) {
  constexpr int RB = KvFmt<FMT>::row(HD), SB = KvFmt<FMT>::scales(HD), TK = HD / 8, N = TK / 4;  // threads of a key, keys of a thread
  constexpr float bias = KvFmt<FMT>::bias;
  const int tid = threadIdx.x, lane = tid & 63, tile = blockIdx.x, h = blockIdx.y;
  const int64_t at = ((int64_t)blockIdx.z * gridDim.y + h) * gridDim.x + tile;
  if (at == 0)  // what fills up the flags
    for (int64_t i = (int64_t)gridDim.x * gridDim.y * gridDim.z + tid; i < a.nflags; i += 256) flags[i] = 0;
  int q0 = 0, lq = 0, len = 0;
  if (lane < a.nseq) {
    q0 = min(max(a.cu_q[lane], 0), a.total_q);
    lq = max(min(max(a.cu_q[lane + 1], 0), a.total_q) - q0, 0);
    len = min(max(a.lens[lane], 0), a.max_len);
  }
  uint64_t many = __ballot((int64_t)lq * a.group > a.over);
  // offsets that overlap can have more such sequences than there is room for: all are done from the codes then
  const bool excess = __popcll(many) > (int)gridDim.z;
  for (int i = 0; i < (int)blockIdx.z; ++i) many &= many - 1;
  const int s = many ? __ffsll((unsigned long long)many) - 1 : 0;
  lq = __builtin_amdgcn_readlane(lq, s), len = many ? __builtin_amdgcn_readlane(len, s) : 0;
  const int first = a.window ? max(max(len - lq, 0) - a.window + 1, 0) : 0;
  if (64 * tile >= len || (64 * tile + 63 < first && 64 * tile >= a.sinks)) {
    if (tid == 0) flags[at] = excess;
    return;
  }
  // neighbouring threads have neighbouring channels, eight each
  const int c = tid % TK;
  uint8_t* const to = out + (((int64_t)blockIdx.z * gridDim.x + tile) * a.kv.heads + h) * (64 * 4 * HD) + tid / TK * (2 * HD) + 16 * c;
  uint2 w[N][2];
  uint16_t scale[N][2];
  uint32_t lost = 0;
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int key = min(64 * tile + 64 / N * n + tid / TK, len - 1);
    const int page = a.table[(int64_t)s * a.ldt + (key >> a.kv.shift)], in = key & ((1 << a.kv.shift) - 1);
    const bool none = page < 0 || page >= a.kv.pages;
    lost |= (uint32_t)none << n;
    const uint8_t* const block = a.kv.data + h * a.kv.block + (uint64_t)(uint32_t)(none ? 0 : page) * (uint32_t)(a.kv.heads * a.kv.block);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const uint8_t* const codes = block + kv_rows_at<FMT, HD>(which, a.kv.shift) + in * RB + c * (RB / TK);
      if constexpr (FMT == DUO_KV_I8)
        w[n][which] = *(const uint2*)codes;
      else
        w[n][which].x = *(const uint32_t*)codes;
      scale[n][which] = *(const uint16_t*)(block + kv_scales_at<FMT, HD>(which, a.kv.shift) + in * SB + c / 4 * 2);
    }
  }
  bool odd = false;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      const bool none = lost >> n & 1;
      const uint16_t sb = scale[n][which];
      int top = sb < 0x7f80 ? sb : 0;
#pragma unroll
      for (int o = 4; o < TK; o <<= 1) top = max(top, __shfl_xor(top, o));
      const int unit = which ? kRowsUnit : 0;
      // (one power of two more than codes have, whose way to numbers goes by 24 times the scale)
      odd |= !none && power_of(__uint_as_float((uint32_t)top << 16) * KvFmt<FMT>::most, kRowsLo + unit, kRowsHi + unit + 1) != 0;
      const float sc = none ? NAN : bf16_bits_to_f32(sb) * (float)(1 << (kRowsBoost - unit)), off = sc * -bias;
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t code = FMT == DUO_KV_I8 ? (e < 4 ? w[n][which].x : w[n][which].y) >> (8 * (e & 3)) & 255u : w[n][which].x >> (4 * e) & 15u;
        v[e] = fmaf((float)code, sc, off);  // exactly
      }
      *(u32x4*)(to + 64 / N * n * (2 * HD) + which * (64 * 2 * HD)) = u32x4{pack_two<true>(v[0], v[1]), pack_two<true>(v[2], v[3]),
                                                                            pack_two<true>(v[4], v[5]), pack_two<true>(v[6], v[7])};
    }
  odd = __syncthreads_or(odd);
  if (tid == 0) flags[at] = odd || excess;
}

// Joins the parts of the block that begins in a share, if it ends in another one: its own
// part (the second of its two places), then the first places of the shares after it.  HD / 4 threads
// per row, blockIdx.y counts the rows by the 1024 / HD that a workgroup takes.  Shares lie on the XCDs
// as in rows_kernel: blocks of equal length begin at shares that are multiples of each other, which
// as blockIdx.x would all be on one XCD (32 tokens on 16384, 64 heads on 8: 67 us for that, 19 so).
template <int HD, bool I4>
__global__ __launch_bounds__(256) void rows_join_kernel(RowsArgs a) {
  constexpr int T = HD / 4;
  const int share = (int)(blockIdx.x & 7) * (int)(gridDim.x >> 3) + (int)(blockIdx.x >> 3);
  const RowsTask task = a.tasks[share];
  const int row = blockIdx.y * (256 / T) + threadIdx.x / T, d = threadIdx.x % T * 4;
  if (task.parts == 0 || row >= task.rows) return;
  const int qi = by(row, a), h = row - qi * a.hg;
  auto part = [&](int i) { return a.parts + (2 * ((int64_t)share + i) + (i == 0)) * rows_part(HD); };
  // eight parts at once, whose outputs, references and sums are all on their way before the first is used
  float top = -INFINITY, sum = 0.f;
  f4 y = {0.f, 0.f, 0.f, 0.f};
  for (int i = 0; i < task.parts; i += 8) {
    float2 ml[8];
    f4 v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float* const p = part(min(i + j, task.parts - 1));
      ml[j] = *(const float2*)(p + kRowsQB * HD + 2 * row);
      v[j] = *(const f4*)(p + row * HD + d);
    }
    float most = top;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = fmaxf(most, ml[j].x);
    const float f = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top - most);
    sum *= f;
    y *= f;
    top = most;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (i + j >= task.parts) break;
      // a part without a finite score holds zeros, or NaN that has to stay
      const float w = ml[j].x == -INFINITY ? ml[j].y : __builtin_amdgcn_exp2f(ml[j].x - top);
      sum += w * ml[j].y;
      y += v[j] * w;
    }
  }
  if (h >= task.heads) return;
  const bool none = task.pos0 + qi < 0;
  const uint2 two = none ? make_uint2(0, 0) : make_uint2(pack_bf16(y[0] / sum, y[1] / sum), pack_bf16(y[2] / sum, y[3] / sum));
  uint16_t* const o = a.O + (int64_t)(task.q0 + qi) * a.ldo + (int64_t)(task.head0 + h) * HD + d;
  if (I4) {  // four of eight channels: c, c + 4, c + 1, c + 5 with c = 0 or 2
    uint16_t* const o8 = o - (d & 4 ? 2 : 0);
    o8[0] = (uint16_t)two.x, o8[4] = (uint16_t)(two.x >> 16);
    o8[1] = (uint16_t)two.y, o8[5] = (uint16_t)(two.y >> 16);
  } else if (a.vec) {
    *(uint2*)o = two;
  } else {
    o[0] = (uint16_t)two.x, o[1] = (uint16_t)(two.x >> 16);
    o[2] = (uint16_t)two.y, o[3] = (uint16_t)(two.y >> 16);
  }
}

}  // namespace duo
