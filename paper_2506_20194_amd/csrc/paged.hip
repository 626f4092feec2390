// Attention of one query per sequence over the paged key-value cache, split over
// the cache's length and joined.
//
// The work is a list of tiles (32 cached tokens in 16 bits, 64 in 8 and 4) of rows,
// a row being one sequence, one K/V head and up to 16 of its query heads.  Tiles of
// all rows are counted through, with some more for what a row costs beside its
// tiles, and every workgroup takes an equal share of the count, wherever rows begin
// and end: sequences of any mix of lengths load the CUs evenly, and no launch size
// depends on the lengths, which only the device knows.  A workgroup's four waves
// take the tiles of a row in turn, each with its own running maximum and sum, and
// join at the row's end; a row that lies in one share is finished there, the parts
// of one that does not go to the workspace and are joined by a second launch.  Where rows
// are many, short ones go four to a workgroup, one for each wave.
//
// A wave computes transposed, with v_mfma_f32_16x16x32_bf16:
//   S^T = K Q^T  (16 keys x 16 heads per instruction): a lane's scores belong to one
//                head, and to the keys 16 b + 4 (lane / 16) + 0..3;
//   O^T = V^T P^T: P^T's fragments are the lane's own probabilities (keys 4 g + 0..3
//                of two blocks of 16), and V^T's take the same keys from the
//                row-major tile with transposing LDS reads.
// Heads that do not fill 16 columns waste matrix work only, of which there is
// plenty: the bound is the cache's bytes.  Tiles go global -> LDS directly, and a
// wave issues the next tile's K as soon as this one's K has been read into registers,
// V likewise, so that one of the two is always in flight and one buffer for each
// suffices (at head_dim 128 and 8 waves per CU 16, 18 or 10 KB for each in 16, 8 and 4 bits).
// A wave needs no other wave for that, so the loop has no barrier.  Probabilities (16 bits), or
// these times V's scales (8 and 4), are rounded to bf16, the matrix instruction's type, for the
// product with V; their sum is of the fp32 ones.  Against 64 bits the root mean square error is
// 0.0016 to 0.0018 of the output's, and 0.0015 to 0.0017 with probabilities in fp32.
//
// 8 and 4 bits.  Codes keep what is added to them: a byte 0..255 converts to a bf16
// number exactly, and a nibble n becomes 128 + n by setting its bits into 0x4300.
// The excess (bias 128, 136) leaves again in the accumulator, which starts at
// -bias sum(q) of the group for S and gets -bias sum(p) from one more MFMA for O.  A
// score is the sum of its groups' products times their scales, in fp32; the scale
// of V goes into the probability before that is rounded to bf16.
//
// Bound: HBM where there is enough to read: 64 sequences of 8192 tokens, 64 heads of 128 on 8,
// 357 us in 16 bits (6.0 TB/s), 205 in 8 (5.6), 122 in 4 (5.0, where the vector work on the
// codes shows); heads of 64 195 (5.5), 114 (5.0) and 65 (4.6), the last 76 with pages of 16,
// whose tiles take the loads that a row's last tile takes.  Short of that what a launch and a row
// begin with: lengths, page numbers and the first K are three trips to memory, 4 us, and the
// join's launch takes another 4 to 5 (one request of 1777 tokens, 32 heads: 10 and 4 us).
// Scalar registers are spilled in every format (35 in 16 bits, 52 to 75 in 8 and 4), into lanes of
// vector registers around the loads in the loop; vector registers are not.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "cache.h"
#include "dma.h"
#include "internal.h"
#include "mfma.h"
#include "pingpong.h"

using namespace duo;
using namespace duo::pp;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) % 16) == 0; }

constexpr int kCols = 16;       // query heads per row
constexpr int kMaxWg = 1024;    // workgroups of a launch, at most
// What a row's start and end cost, in tiles.  Eight sequences of 1 to 131072 tokens in 4 bits, 64
// heads on 8: 73 us with 4, 55 with 8, 51 with 10 and 14; 48 of up to 8192 in 8 bits: 51, 46, 47, 47.
constexpr int kRowCost = 10;
// Smallest share, in tiles: one sequence of 4096 tokens in 4 bits 13.3 us, 17.3 with 16; with 4
// as with 8, for twice the parts.
constexpr int kMinShare = 8;
// Tiles of a row that one wave does alone where rows are many: 512 sequences of 100 tokens in 4
// bits, 64 heads on 8, 68 us with 0, 32 with 4 and 8; 128 of 256 tokens in 16 bits, 32 on 8, 26 us
// with 0 and 4, 33 with 8.  Where rows are few four waves on one are shorter: 4 sequences of 250 tokens
// in 8 bits, 64 on 8, 11 us, and 16 with a wave alone.
constexpr int kShort = 4;
constexpr int kMinKeys = 32;    // tokens of the smallest tile

template <int FMT, int HD>
struct PagedGeo {
  static constexpr int KEYS = FMT == DUO_KV_BF16 ? 32 : 64;
  static constexpr int NB = KEYS / 16;                     // blocks of 16 keys
  static constexpr int CK = HD / 32;                       // MFMA steps over head_dim, groups with a scale
  static constexpr int RB = KvFmt<FMT>::row(HD), CH = RB / 16;
  static constexpr int RPL = 64 / CH, NL = KEYS / RPL;     // rows per wave-wide load, loads per operand
  static constexpr int SB = KvFmt<FMT>::scales(HD);
  static constexpr int NS = (KEYS * SB + 255) / 256;       // loads of scales per operand
  static constexpr int ROWS = KEYS * RB;                   // bytes of one operand's rows
  static constexpr int WAVE = 2 * (ROWS + 2 * NS * 256);   // LDS of a wave; scales have two buffers
  static constexpr int OLD = HD + 4;                       // row stride of the join's fp32 outputs
  static_assert(kCols * OLD * 4 <= WAVE, "the join uses a wave's tile space");
  // Workgroups per CU: two where LDS holds no more, or (4 bits, head_dim 128) the vector registers:
  // with three some of them are spilled in the loop (8 sequences of up to 131072 tokens 66 us; 52).
  static constexpr int WGS = 4 * WAVE >= 40960 ? 2 : FMT != DUO_KV_BF16 ? 3 : 4;
};

// The rows to do, and into how many shares at most.
struct PagedWork {
  const int32_t* lens;
  int nseq, max_len, rows;  // rows per sequence
  int per;                  // sequences per bucket of the count: ceil(nseq / 64)
  int many;                 // rows enough for every share: short ones go four to a workgroup
};

// A row that begins in a share and ends in another one: the join's task.  parts = 0: none.
struct Task {
  int seq, row, parts, pad;
};

__device__ inline int seq_len(const PagedWork& w, int s) { return min(max(w.lens[s], 0), w.max_len); }

// Tiles, and what counts for one row of them.
template <int KEYS>
__device__ inline int tiles_of(int len) { return (len + KEYS - 1) / KEYS; }

// The rows of a sequence of `tiles` tiles: `units` of `cost` each.  A unit is a row, or four
// rows, one for each wave, where they are short and many.
struct Units {
  int tiles, cost, units;
  bool quad;
  __device__ Units(int tiles, const PagedWork& w) : tiles(tiles) {
    quad = w.many && tiles <= kShort;
    units = tiles == 0 ? 0 : quad ? (w.rows + 3) / 4 : w.rows;
    cost = (quad ? 4 * tiles : tiles) + kRowCost;
  }
};

__device__ inline uint64_t div64(uint64_t a, uint32_t b) { return a >> 32 ? a / b : (uint32_t)a / b; }

// The count cut into n shares as equal as whole numbers allow: share i begins at
// i size + min(i, more).
struct Shares {
  int64_t size;
  int more, n;
  __device__ Shares(int64_t total, int most) {
    n = (int)min((int64_t)most, (total + kMinShare - 1) / kMinShare);
    size = n ? (int64_t)div64((uint64_t)total, (uint32_t)n) : 0;
    more = (int)(total - size * n);
  }
  __device__ int64_t begin(int i) const { return i * size + min(i, more); }
  __device__ int of(int64_t u) const {  // size < 2^31: fewer than 2^31 of anything in 2^10 shares
    const int64_t cut = more * (size + 1);
    return u < cut ? (int)div64((uint64_t)u, (uint32_t)size + 1) : more + (int)div64((uint64_t)(u - cut), (uint32_t)size);
  }
};

__device__ inline int64_t lane64(int64_t v, int l) {
  return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), l) << 32 |
                   (uint32_t)__builtin_amdgcn_readlane((int)v, l));
}

// Cost of the sequences up to the end of this lane's bucket of `per`.  Every wave counts for
// itself: no barrier, and no wave waits for another.  *len: this lane's sequence, where a
// bucket is one.
template <int KEYS>
__device__ inline int64_t count_rows(const PagedWork& w, int* len) {
  const int lane = threadIdx.x & 63;
  int64_t n = 0;
  *len = 0;
#pragma unroll 4
  for (int i = 0; i < w.per; ++i) {
    const int64_t s = (int64_t)lane * w.per + i;
    *len = s < w.nseq ? seq_len(w, (int)s) : 0;
    const Units x(tiles_of<KEYS>(*len), w);
    n += (int64_t)x.cost * x.units;
  }
  // running sum over the lanes: within rows of 16, then over the rows
#define DUO_UP(o)                                                                                        \
  n += (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_update_dpp(0, (int)(n >> 32), 0x110 + o, 0xf, 0xf, true) << 32 | \
                 (uint32_t)__builtin_amdgcn_update_dpp(0, (int)n, 0x110 + o, 0xf, 0xf, true))
  DUO_UP(1);
  DUO_UP(2);
  DUO_UP(4);
  DUO_UP(8);
#undef DUO_UP
  const int64_t r0 = lane64(n, 15), r1 = r0 + lane64(n, 31), r2 = r1 + lane64(n, 47);
  return n + (lane < 16 ? 0 : lane < 32 ? r0 : lane < 48 ? r1 : r2);
}

// max over the four lanes that hold one column
__device__ __forceinline__ float col_max(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float col_sum(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The value of the lane eight places on, within groups of sixteen lanes.
__device__ __forceinline__ float ror8(float v) {
  return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x128, 0xf, 0xf, false));
}

__device__ __forceinline__ float lo16(uint32_t v) { return __uint_as_float(v << 16); }
__device__ __forceinline__ float hi16(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }

// Eight codes as bf16 with their bias: bytes in order; nibbles j and j + 4 in register j.
__device__ __forceinline__ u32x4 widen8(uint32_t a, uint32_t b) {
  auto f = [](uint32_t v, int i) { return (float)(v >> (8 * i) & 255u); };
  return u32x4{pack_bf16(f(a, 0), f(a, 1)), pack_bf16(f(a, 2), f(a, 3)), pack_bf16(f(b, 0), f(b, 1)),
               pack_bf16(f(b, 2), f(b, 3))};
}
__device__ __forceinline__ u32x4 widen4(uint32_t a) {
  u32x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = (a >> (4 * j) & 0x000f000fu) | 0x43004300u;
  return r;
}

// Position of 16-byte chunk c of row r in an LDS tile, so that the rows that one
// fragment read touches lie in different banks.
template <int FMT, int CH>
__device__ __forceinline__ int k_at(int r, int c) {
  return c ^ (CH == 16 ? r & 15 : CH == 8 ? r >> 1 & 7 : CH == 4 ? r >> 2 & 3 : r >> 3 & 1);
}
template <int FMT, int CH>
__device__ __forceinline__ int v_at(int r, int c) {
  if constexpr (FMT == DUO_KV_BF16)  // 8 keys x 32 bytes at once
    return c ^ (CH == 16 ? 2 * (r & 7) : 2 * (r >> 1 & 3));
  else if constexpr (CH == 8)        // keys 0..7 and 16..23, or 8..15 and 24..31, x 16 bytes
    return c ^ ((r >> 1 & 3) | (r >> 2 & 4));
  else if constexpr (CH == 4)
    return c ^ ((r >> 2 & 1) | (r >> 3 & 2));
  else
    return c ^ (r >> 4 & 1);
}

// PAIR (8 and 4 bits, at most 8 heads): the columns that would stay empty take the second
// half of the tile's keys.  A block of keys of each half is multiplied with the queries in
// its half of the columns, both into one accumulator, and what follows for a score
// (scales, maximum, exponential, rounding), the larger part of the vector work, is done
// for two keys at once; the halves of a column's pair meet at the join.  64 sequences of 8192
// tokens, 64 heads on 8: 214 us without and 206 with in 8 bits, 133 and 121 in 4.
template <int FMT, int HD, bool PAIR>
__global__ __launch_bounds__(256, (PagedGeo<FMT, HD>::WGS)) void paged_kernel(
    const uint16_t* __restrict__ Q, int64_t ldq, KvGeo kv, const int32_t* __restrict__ table, int64_t ldt, PagedWork work,
    int group, int cols, float cexp, uint32_t flip, uint16_t* __restrict__ O, int64_t ldo, Task* __restrict__ tasks,
    float* __restrict__ part, int vec) {
  using G = PagedGeo<FMT, HD>;
  constexpr int KEYS = G::KEYS, NB = G::NB, CK = G::CK, RB = G::RB, CH = G::CH, RPL = G::RPL, NL = G::NL, NS = G::NS;
  constexpr int NK = NL + NS;  // loads per operand and tile
  constexpr bool QUANT = FMT != DUO_KV_BF16;
  constexpr int XB = PAIR ? NB / 2 : NB;  // blocks of 16 keys in a lane's scores
  static_assert(QUANT || !PAIR, "");
  constexpr float BIAS = FMT == DUO_KV_I8 ? 128.f : 136.f;
  extern __shared__ __attribute__((aligned(16))) uint8_t lsm[];
  __shared__ float jm[4][kCols], jl[4][kCols];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l16 = lane & 15, g = lane >> 4;
  const int col = PAIR ? l16 & 7 : l16, half = PAIR ? l16 >> 3 : 0;  // this lane's head, and half of the keys

  int my_len;
  const int64_t upto = count_rows<KEYS>(work, &my_len);
  const Shares shares(lane64(upto, 63), gridDim.x);
  int64_t u = shares.begin(blockIdx.x);
  const int64_t u1 = (int)blockIdx.x < shares.n ? shares.begin(blockIdx.x + 1) : u;
  if (tid == 0 && tasks) tasks[blockIdx.x].parts = 0;
  auto len_of = [&](int s) {
    return work.per == 1 ? __builtin_amdgcn_readlane(my_len, s) : __builtin_amdgcn_readfirstlane(seq_len(work, s));
  };
  // sequences without tokens
  for (int s = blockIdx.x; s < work.nseq; s += gridDim.x)
    if (len_of(s) == 0)
      for (int e = tid; e < group * kv.heads * HD; e += 256) O[(int64_t)s * ldo + e] = 0;
  if (u >= u1) return;
  // the bucket that u lies in: the first whose end lies behind it
  const int at_bucket = __ffsll((unsigned long long)__ballot(upto > u)) - 1;
  int64_t before = at_bucket ? lane64(upto, at_bucket - 1) : 0;  // cost of the sequences before s
  uint8_t* const sK = lsm + wave * G::WAVE;
  uint8_t* const sV = sK + G::ROWS;
  uint8_t* const sS = sV + G::ROWS;  // scales: [parity of the tile's turn][K, V]

  for (int s = at_bucket * work.per; u < u1; ++s) {
    const int len = len_of(s);
    const Units x(tiles_of<KEYS>(len), work);
    const int tiles = x.tiles, cost = x.cost;
    const int64_t start = before;
    before += (int64_t)cost * x.units;
    if (before <= u) continue;
    const int32_t* const pages = table + (int64_t)s * ldt;
    const int last_page = (len - 1) >> kv.shift;
    while (u < u1 && u < before) {
      // one row, or what of it is in this share
      int row = (int)div64((uint64_t)(u - start), (uint32_t)cost);
      const int at = (int)(u - start - (int64_t)row * cost);
      const int here = (int)min((int64_t)(cost - at), u1 - u);
      int t0 = max(at - kRowCost, 0), t1 = max(at + here - kRowCost, 0);
      const int64_t row_end = u + (cost - at);
      u += here;
      int t = t0 + wave, step = 4;  // this wave's tiles
      if (x.quad) {  // whole in the share that it begins in
        if (at > 0) continue;
        row = 4 * row + wave;
        if (row >= work.rows) continue;
        t = t0 = 0;
        t1 = tiles;
        step = 1;
      }
      if (t0 >= t1) continue;
      const int h = row % kv.heads, c0 = row / kv.heads * kCols;  // K/V head, first of its query heads
      const int nc = min(cols, group - c0);
      const uint16_t* const q = Q + (int64_t)s * ldq + (h * group + c0) * HD;
      const uint8_t* const block0 = kv.data + h * kv.block;
      const uint32_t page_bytes = (uint32_t)(kv.heads * kv.block);

      // 64 pages of the table in one register, the next 64 in another
      bool bad = false;
      int win = (t * KEYS >> kv.shift) & ~3;  // a tile's pages, four at most, lie in one window
      auto ids = [&](int p) {
        int id = pages[min(p + lane, last_page)];
        const bool out = id < 0 || id >= kv.pages;
        bad |= out;
        return out ? 0 : id;
      };
      int pid = ids(win), nid = ids(win + 64);
      u32x4 qf[CK];
#pragma unroll
      for (int c = 0; c < CK; ++c) qf[c] = *(const u32x4*)(q + min(col, nc - 1) * HD + 32 * c + 8 * g);
#pragma unroll
      for (int c = 0; c < CK; ++c) asm volatile("" : "+v"(qf[c]));  // waited for here, and not behind the tiles
      // this wave's loads of tile t's K (which = 0) or V rows and scales; K first
      auto issue = [&](int t, auto which_c, const uint8_t* to_rows, const uint8_t* to_scales) __attribute__((always_inline)) {
        constexpr int which = decltype(which_c)::value;
        const int k0 = t * KEYS;
        const uint32_t rows = __builtin_amdgcn_readfirstlane(lds_addr(to_rows));
        const uint32_t scales = __builtin_amdgcn_readfirstlane(lds_addr(to_scales));
        if (which == 0 && k0 >> kv.shift >= win + 64) {  // four tiles never reach further than the next window
          pid = nid;
          win += 64;
          nid = ids(win + 64);
        }
        const int rows_at = kv_rows_at<FMT, HD>(which, kv.shift), scales_at = kv_scales_at<FMT, HD>(which, kv.shift);
        const int mask = (1 << kv.shift) - 1;
        auto chunk = [&](int r) {
          const int p = lane % CH;
          return 16 * (which ? v_at<FMT, CH>(r, p) : k_at<FMT, CH>(r, p));
        };
        if (k0 + KEYS <= len && 1 << kv.shift >= KEYS) {
          // whole tile in one page: its rows and scales are runs of bytes
          const int id = __builtin_amdgcn_readlane(pid, (k0 >> kv.shift) - win);
          const uint8_t* const at = block0 + (uint64_t)(uint32_t)id * page_bytes;
          const int in = k0 & mask;
          uint32_t off[NL];
#pragma unroll
          for (int i = 0; i < NL; ++i) off[i] = lane / CH * RB + chunk(i * RPL + lane / CH);
          dma16_run<NL>(at + (rows_at + in * RB), off, rows);
          if constexpr (QUANT) {
#pragma unroll
            for (int i = 0; i < NS; ++i) dma4(at + (scales_at + in * G::SB + 256 * i), lane * 4, scales + i * 256);
          }
        } else if (k0 + KEYS <= len && RPL <= 16) {
          // whole tile in several pages: each group of 16 keys lies in one, the same for all lanes
          const uint8_t* base[NB];
          int in[NB];
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const int key = k0 + 16 * b;
            const int id = __builtin_amdgcn_readlane(pid, (key >> kv.shift) - win);
            base[b] = block0 + (uint64_t)(uint32_t)id * page_bytes;
            in[b] = key & mask;
          }
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const int r = i * RPL + lane / CH, b = i * RPL / 16;
            const uint8_t* at = base[b] + (rows_at + in[b] * RB);
            dma16(at, (uint32_t)((r & 15) * RB + chunk(r)), rows + i * 1024);
          }
          if constexpr (QUANT) {
#pragma unroll
            for (int i = 0; i < NS; ++i) {
              constexpr int BPL = 256 / (16 * G::SB);  // blocks of 16 keys per load
              const int bl = lane * 4 / (16 * G::SB);
              const uint8_t* at = base[i * BPL] + (scales_at + in[i * BPL] * G::SB);
#pragma unroll
              for (int b = 1; b < BPL; ++b) {
                const uint8_t* x = base[i * BPL + b] + (scales_at + in[i * BPL + b] * G::SB);
                at = bl == b ? x : at;
              }
              dma4(at + lane * 4 % (16 * G::SB), scales + i * 256);
            }
          }
        } else {
          // the row's last tile: rows past its end are taken from its last token, and
          // neither their scores nor (below) their values enter
          auto place = [&](int r) {
            const int key = min(k0 + r, len - 1);
            const int id = __shfl(pid, (key >> kv.shift) - win);
            return std::make_pair(block0 + (uint64_t)(uint32_t)id * page_bytes, key & mask);
          };
#pragma unroll 1
          for (int i = 0; i < NL; ++i) {
            const int r = i * RPL + lane / CH;
            const auto [b, in] = place(r);
            dma16(b + rows_at + in * RB + chunk(r), rows + i * 1024);
          }
          if constexpr (QUANT) {
#pragma unroll 1
            for (int i = 0; i < NS; ++i) {
              const int e = i * 256 + lane * 4;
              const auto [b, in] = place(e / G::SB);
              dma4(b + scales_at + in * G::SB + e % G::SB, scales + i * 256);
            }
          }
        }
      };
      constexpr std::integral_constant<int, 0> kK{};
      constexpr std::integral_constant<int, 1> kV{};

      float m = -INFINITY, mc = -INFINITY, l = 0.f;  // of this lane's column; l of its keys alone
      f4 o[2 * CK];
#pragma unroll
      for (int d = 0; d < 2 * CK; ++d) o[d] = f4{0.f, 0.f, 0.f, 0.f};

      if (t < t1) {
        issue(t, kK, sK, sS);
        issue(t, kV, sV, sS + NS * 256);
      }
      // Q^T's fragments, heads past the last as zeros; -bias sum(q) of every group
      float qs[CK];
      u32x4 qh[CK];  // of the second half's columns
#pragma unroll
      for (int c = 0; c < CK; ++c) {
        u32x4 v = qf[c];
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = col < nc ? v[j] ^ flip : 0u;
        if constexpr (QUANT) {
          float t = 0.f;
#pragma unroll
          for (int j = 0; j < 4; ++j) t += lo16(v[j]) + hi16(v[j]);
          qs[c] = -BIAS * col_sum(t);
        }
        if constexpr (FMT == DUO_KV_I4)  // channels j and j + 4 together, as widen4 gives them
          v = u32x4{(v[0] & 0xffffu) | v[2] << 16, v[0] >> 16 | (v[2] & 0xffff0000u), (v[1] & 0xffffu) | v[3] << 16,
                    v[1] >> 16 | (v[3] & 0xffff0000u)};
#pragma unroll
        for (int j = 0; j < 4; ++j) qf[c][j] = half ? 0u : v[j], qh[c][j] = half ? v[j] : 0u;
      }
      for (uint8_t* sc = sS; t < t1; t += step) {
        const bool more = t + step < t1;
        uint8_t* const sn = sc == sS ? sS + 2 * NS * 256 : sS;  // the next tile's scales
        wait_vm<NK>();  // K of this tile
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        // ---- scores
        float x[XB][4];
        if constexpr (!QUANT) {
          u32x4 kf[NB][CK];
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int c = 0; c < CK; ++c)
              kf[b][c] = *(const u32x4*)(sK + (16 * b + l16) * RB + 16 * k_at<FMT, CH>(16 * b + l16, 4 * c + g));
          wait_lds<0>();
          if (more) issue(t + step, kK, sK, sn);
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            f4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < CK; ++c) a = mma_bf16(kf[b][c], qf[c], a);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[b][r] = a[r];
          }
        } else {
          uint2 kr[NB][CK];
#pragma unroll
          for (int b = 0; b < NB; ++b) {
            const int r = 16 * b + l16;
#pragma unroll
            for (int c = 0; c < CK; ++c) {
              if constexpr (FMT == DUO_KV_I8)
                kr[b][c] = *(const uint2*)(sK + r * RB + 16 * k_at<FMT, CH>(r, 2 * c + g / 2) + 8 * (g & 1));
              else
                kr[b][c].x = *(const uint32_t*)(sK + r * RB + 16 * k_at<FMT, CH>(r, c) + 4 * g);
            }
          }
          wait_lds<0>();
          if (more) issue(t + step, kK, sK, sn);
          auto widen = [](const uint2& v) { return FMT == DUO_KV_I8 ? widen8(v.x, v.y) : widen4(v.x); };
#pragma unroll
          for (int b = 0; b < XB; ++b) {
            uint32_t ks[2 * CK];  // scales of the lane's four keys
#pragma unroll
            for (int j = 0; j < 2 * CK; j += 4)
              *(u32x4*)&ks[j] = *(const u32x4*)(sc + (32 * half + 16 * b + 4 * g) * G::SB + 4 * j);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[b][r] = 0.f;
#pragma unroll
            for (int c = 0; c < CK; ++c) {
              f4 a = mma_bf16(widen(kr[b][c]), qf[c], f4{qs[c], qs[c], qs[c], qs[c]});
              if constexpr (PAIR) a = mma_bf16(widen(kr[b + XB][c]), qh[c], a);
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const uint32_t w = ks[(r * CK + c) / 2];
                x[b][r] = fmaf((r * CK + c) & 1 ? hi16(w) : lo16(w), a[r], x[b][r]);
              }
            }
          }
        }
        // ---- probabilities relative to the running maximum
        const int left = len - t * KEYS - 32 * half - 4 * g;  // tokens of the row from this lane's first key on
#pragma unroll
        for (int b = 0; b < XB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[b][r] = 16 * b + r < left ? x[b][r] : -INFINITY;
        float mt = x[0][0];
#pragma unroll
        for (int b = 0; b < XB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) mt = fmaxf(mt, x[b][r]);
        mt = col_max(mt);
        if (__any(mt > m)) {
          const float mn = fmaxf(m, mt);
          const float mcn = mn == -INFINITY ? -INFINITY : mn * cexp;
          const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - mcn);
          m = mn;
          mc = mcn;
          l *= f;
#pragma unroll
          for (int d = 0; d < 2 * CK; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) o[d][r] *= f;
        }
        const float base = m == -INFINITY ? 0.f : mc;
#pragma unroll
        for (int b = 0; b < XB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) x[b][r] = __builtin_amdgcn_exp2f(fmaf(x[b][r], cexp, -base));
#pragma unroll
        for (int b = 0; b < XB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) l += x[b][r];
        // ---- times V
        if (more)
          wait_vm<NK>();  // V of this tile; K of the next may be in flight
        else
          wait_vm<0>();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!QUANT) {
          typedef __attribute__((address_space(3))) s16v4 lds4;
          u32x4 vf[2 * CK];
#pragma unroll
          for (int d = 0; d < 2 * CK; ++d) {
            // 16 lanes: four keys (by l16 / 4) x 16 channels
            const int r0 = 4 * g + (l16 >> 2), r1 = r0 + 16, c = 2 * d + (l16 >> 1 & 1), e = 8 * (l16 & 1);
            const s16v4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(sV + r0 * RB + 16 * v_at<FMT, CH>(r0, c) + e));
            const s16v4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4*)(sV + r1 * RB + 16 * v_at<FMT, CH>(r1, c) + e));
            __builtin_memcpy(&vf[d], &a, 8);
            __builtin_memcpy((char*)&vf[d] + 8, &b, 8);
          }
          wait_lds<0>();
          if (more) issue(t + step, kV, sV, sn + NS * 256);
          if (t * KEYS + KEYS > len) {
            // copies of the last token behind the row's end: their probability is 0, and 0 times
            // an infinite value would be NaN (codes are finite, and a scale that is not is NaN)
            int rest = left;
            asm volatile("" : "+v"(rest));  // compared here: the scores' comparisons would be kept for it in the loop
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int key = 16 * (j >> 1) + 2 * (j & 1);  // the register's two keys: this one and the next
              const uint32_t keep = (key < rest ? 0xffffu : 0u) | (key + 1 < rest ? 0xffff0000u : 0u);
#pragma unroll
              for (int d = 0; d < 2 * CK; ++d) vf[d][j] &= keep;
            }
          }
          const u32x4 pf = {pack_bf16(x[0][0], x[0][1]), pack_bf16(x[0][2], x[0][3]), pack_bf16(x[1][0], x[1][1]),
                            pack_bf16(x[1][2], x[1][3])};
#pragma unroll
          for (int d = 0; d < 2 * CK; ++d) o[d] = mma_bf16(vf[d], pf, o[d]);
        } else {
          typedef int v2i __attribute__((ext_vector_type(2)));
          typedef __attribute__((address_space(3))) v2i lds2;
          v2i vr[FMT == DUO_KV_I8 ? 2 : 1][2 * CK];
#pragma unroll
          for (int d = 0; d < 2 * CK; ++d) {
            if constexpr (FMT == DUO_KV_I8) {
#pragma unroll
              for (int st = 0; st < 2; ++st) {  // 16 lanes: eight keys (by l16 / 2) x 16 channels
                const int i = l16 >> 1, r = 32 * st + (i < 4 ? 4 * g + i : 12 + 4 * g + i);
                vr[st][d] = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
                    (lds2*)(sV + r * RB + 16 * v_at<FMT, CH>(r, d) + 8 * (l16 & 1)));
              }
            } else {  // 16 lanes: sixteen keys x 16 channels
              const int i = l16 & 7, r = 32 * (l16 >> 3) + (i < 4 ? 4 * g + i : 12 + 4 * g + i);
              vr[0][d] =
                  __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds2*)(sV + r * RB + 16 * v_at<FMT, CH>(r, d / 2) + 8 * (d & 1)));
            }
          }
          wait_lds<0>();
          if (more) issue(t + step, kV, sV, sn + NS * 256);
          const uint32_t nb = pack_bf16(-BIAS, -BIAS);
          const u32x4 bias = {nb, nb, nb, nb};
          // probabilities times scales of the 32 keys of blocks 2 st and 2 st + 1, by groups of channels
          auto weigh = [&](int st, u32x4 (&pf)[CK]) __attribute__((always_inline)) {
            uint32_t vs[2][2 * CK];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
              for (int j = 0; j < 2 * CK; j += 4)
                *(u32x4*)&vs[b][j] =
                    *(const u32x4*)(sc + NS * 256 + (32 * (PAIR ? half : st) + 16 * b + 4 * g) * G::SB + 4 * j);
#pragma unroll
            for (int c = 0; c < CK; ++c) {
              float p[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const int r = e & 3;
                const uint32_t w = vs[e >> 2][(r * CK + c) / 2];
                p[e] = x[(PAIR ? 0 : 2 * st) + (e >> 2)][r] * ((r * CK + c) & 1 ? hi16(w) : lo16(w));
              }
#pragma unroll
              for (int j = 0; j < 4; ++j)
                pf[c][j] = FMT == DUO_KV_I8 ? pack_bf16(p[2 * j], p[2 * j + 1]) : pack_bf16(p[j], p[j + 4]);
            }
          };
          u32x4 pf[CK];
          if constexpr (PAIR) weigh(0, pf);
#pragma unroll
          for (int st = 0; st < 2; ++st) {
            if constexpr (!PAIR) weigh(st, pf);
#pragma unroll
            for (int c = 0; c < CK; ++c) {
              u32x4 ph = pf[c];
              if constexpr (PAIR)
#pragma unroll
                for (int j = 0; j < 4; ++j) ph[j] = half == st ? ph[j] : 0u;
#pragma unroll
              for (int d = 2 * c; d < 2 * c + 2; ++d) {
                const u32x4 vf = FMT == DUO_KV_I8 ? widen8((uint32_t)vr[st][d][0], (uint32_t)vr[st][d][1])
                                                  : widen4((uint32_t)vr[0][d][st]);
                o[d] = mma_bf16(vf, ph, mma_bf16(bias, ph, o[d]));
              }
            }
          }
        }
        sc = sn;
      }
      // ---- the four waves joined: outputs relative to the largest maximum, added up in LDS
#pragma unroll
      for (int d = 0; d < 2 * CK; ++d) asm volatile("s_nop 7" : "+v"(o[d]));  // the last products have been written
      if (__any(bad)) l = NAN;
      l = col_sum(l);
      if (x.quad) {
        // alone: the halves of the keys joined in registers, and written
        if constexpr (PAIR) {
          const float mo = ror8(mc), top = fmaxf(mc, mo);
          // a half without a finite score holds zeros, or NaN that has to stay
          const float f = mc == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - top);
          l = mc == -INFINITY ? l : l * f;
          l += ror8(l);
#pragma unroll
          for (int d = 0; d < 2 * CK; ++d)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float v = o[d][r] * f;
              o[d][r] = v + ror8(v);
            }
        }
        if (half == 0 && col < nc) {
          uint16_t* const y = O + (int64_t)s * ldo + (h * group + c0 + col) * HD + 4 * g;
#pragma unroll
          for (int d = 0; d < 2 * CK; ++d) {
            const uint32_t y0 = pack_bf16(o[d][0] / l, o[d][1] / l), y1 = pack_bf16(o[d][2] / l, o[d][3] / l);
            if (vec) {
              *(uint32_t*)(y + 16 * d) = y0;
              *(uint32_t*)(y + 16 * d + 2) = y1;
            } else {
              y[16 * d] = (uint16_t)y0, y[16 * d + 1] = (uint16_t)(y0 >> 16);
              y[16 * d + 2] = (uint16_t)y1, y[16 * d + 3] = (uint16_t)(y1 >> 16);
            }
          }
        }
        continue;
      }
      if (g == 0) jm[wave][l16] = mc, jl[wave][l16] = l;
      __syncthreads();
      auto largest = [&](int c) {
        float v = fmaxf(fmaxf(jm[0][c], jm[1][c]), fmaxf(jm[2][c], jm[3][c]));
        if constexpr (PAIR) v = fmaxf(v, fmaxf(fmaxf(jm[0][c + 8], jm[1][c + 8]), fmaxf(jm[2][c + 8], jm[3][c + 8])));
        return v;
      };
      const float top = largest(col);
      {
        const float f = mc == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mc - top);
        float* y = (float*)sK + l16 * G::OLD + 4 * g;
#pragma unroll
        for (int d = 0; d < 2 * CK; ++d) {
          // a wave without a finite score holds zeros, or NaN that has to stay
          const f4 v = {o[d][0] * f, o[d][1] * f, o[d][2] * f, o[d][3] * f};
          *(f4*)(y + 16 * d) = v;
        }
      }
      __syncthreads();
      // a share has at most one row that began before it, and one that ends after it
      const bool whole = t0 == 0 && t1 == tiles;
      float* const ps = part + (2 * (int64_t)blockIdx.x + (t0 == 0)) * cols * (HD + 2);
      if (!whole && t0 == 0 && tid == 0) {
        tasks[blockIdx.x] = Task{s, row, shares.of(row_end - 1) - (int)blockIdx.x + 1, 0};
      }
      for (int e = tid; e < nc * (HD / 2); e += 256) {
        const int c = e / (HD / 2), d = e % (HD / 2) * 2;
        const float big = largest(c);
        float sum = 0.f, v0 = 0.f, v1 = 0.f;
#pragma unroll
        for (int i = 0; i < (PAIR ? 8 : 4); ++i) {
          const int w = i & 3, k = c + 8 * (i >> 2);
          const float f = jm[w][k] == -INFINITY ? (jl[w][k] == 0.f ? 0.f : jl[w][k]) : __builtin_amdgcn_exp2f(jm[w][k] - big);
          sum += jl[w][k] * f;
          const float* y = (const float*)(lsm + w * G::WAVE) + k * G::OLD + d;
          v0 += y[0];
          v1 += y[1];
        }
        if (whole) {
          uint16_t* const y = O + (int64_t)s * ldo + (h * group + c0 + c) * HD + d;
          const uint32_t two = pack_bf16(v0 / sum, v1 / sum);
          if (vec)
            *(uint32_t*)y = two;
          else
            y[0] = (uint16_t)two, y[1] = (uint16_t)(two >> 16);
        } else {
          float* const y = ps + c * (HD + 2);
          *(float2*)(y + d) = make_float2(v0, v1);
          if (d == 0) *(float2*)(y + HD) = make_float2(big, sum);
        }
      }
      __syncthreads();
    }
  }
}

// Joins the parts of the rows that lie in several shares: one workgroup for two heads of
// the row that begins in share blockIdx.x, if any does and ends in another: its own part
// (the second of its two places), then the first places of the shares after it.
template <int HD>
__global__ __launch_bounds__(256) void paged_join_kernel(const Task* __restrict__ tasks, const float* __restrict__ part,
                                                         int kv_heads, int group, int cols, uint16_t* __restrict__ O,
                                                         int64_t ldo, int vec) {
  constexpr int T = HD / 4, NP = 128 / T;  // threads per part and head, parts at once
  __shared__ float wt[2][kMaxWg], ls[2][kMaxWg];
  __shared__ float red[2][2][2];
  __shared__ float acc[2][NP][HD];
  const Task task = tasks[blockIdx.x];
  if (task.parts == 0) return;
  const int tid = threadIdx.x & 127, j = threadIdx.x >> 7;  // j: which of the two heads
  const int row = task.row, np = task.parts, h = row % kv_heads, c0 = row / kv_heads * kCols;
  const int c = blockIdx.y * 2 + j, live = c < min(cols, group - c0);
  const int64_t stride = (int64_t)cols * (HD + 2);
  const float* const p0 = part + 2 * (int64_t)blockIdx.x * stride + (live ? c : 0) * (HD + 2);
  auto at = [&](int i) { return p0 + (i ? 2 * i : 1) * stride; };
  // the first parts' outputs are on their way while the weights are found
  const int d = tid % T * 4, k = tid / T;
  constexpr int EARLY = 4;
  f4 first[EARLY];
  auto load = [&](int i) {
    const float2 v0 = *(const float2*)(at(i) + d), v1 = *(const float2*)(at(i) + d + 2);
    return f4{v0.x, v0.y, v1.x, v1.y};
  };
#pragma unroll
  for (int i = 0; i < EARLY; ++i) first[i] = load(min(k + i * NP, np - 1));
  // weights: exp of each part's maximum relative to the largest, and the sum of all
  float top = -INFINITY;
  for (int i = tid; i < np; i += 128) {
    const float2 ml = *(const float2*)(at(i) + HD);
    wt[j][i] = ml.x;
    ls[j][i] = ml.y;
    top = fmaxf(top, ml.x);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  if (tid % 64 == 0) red[0][j][tid >> 6] = top;
  __syncthreads();
  top = fmaxf(red[0][j][0], red[0][j][1]);
  float sum = 0.f;
  for (int i = tid; i < np; i += 128) {
    const float m = wt[j][i], l = ls[j][i];
    const float f = m == -INFINITY ? (l == 0.f ? 0.f : l) : __builtin_amdgcn_exp2f(m - top);
    wt[j][i] = f;
    sum += f * l;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  if (tid % 64 == 0) red[1][j][tid >> 6] = sum;
  __syncthreads();
  sum = red[1][j][0] + red[1][j][1];
  f4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < EARLY; ++i)
    if (k + i * NP < np) a += first[i] * wt[j][k + i * NP];
#pragma unroll 4
  for (int i = k + EARLY * NP; i < np; i += NP) a += load(i) * wt[j][i];
  *(f4*)&acc[j][k][d] = a;
  __syncthreads();
  if (tid < HD / 2 && live) {
    float y0 = 0.f, y1 = 0.f;
#pragma unroll
    for (int i = 0; i < NP; ++i) y0 += acc[j][i][2 * tid], y1 += acc[j][i][2 * tid + 1];
    const uint32_t two = pack_bf16(y0 / sum, y1 / sum);
    uint16_t* const y = O + (int64_t)task.seq * ldo + (h * group + c0 + c) * HD + 2 * tid;
    if (vec)
      *(uint32_t*)y = two;
    else
      y[0] = (uint16_t)two, y[1] = (uint16_t)(two >> 16);
  }
}

// Workgroups for rows of at most `tiles` tiles: no more than smallest shares.
int64_t paged_wgs(double rows, int64_t tiles, int most) {
  const double cost = tiles ? rows * (double)(tiles + kRowCost) / kMinShare : 1.0;
  return cost < most ? std::max<int64_t>(1, (int64_t)std::ceil(cost)) : most;
}

}  // namespace

extern "C" {

size_t duo_attention_paged_workspace_size(int64_t nseq, int64_t heads, int64_t kv_heads, int64_t head_dim,
                                          int64_t max_len) {
  if (nseq < 1 || heads < 1 || kv_heads < 1 || heads % kv_heads || max_len < 1 || (head_dim != 64 && head_dim != 128))
    return 0;
  const int64_t group = heads / kv_heads, cols = std::min<int64_t>(group, kCols);
  // one task and two parts per workgroup
  const int64_t wgs = paged_wgs((double)nseq * (double)(kv_heads * cdiv(group, kCols)), cdiv(max_len, kMinKeys), kMaxWg);
  return align_up(wgs * sizeof(Task)) + align_up((size_t)(2 * wgs * cols * (head_dim + 2)) * sizeof(float));
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
  const int64_t group = heads / g.heads, cols = std::min<int64_t>(group, kCols), rows = g.heads * cdiv(group, kCols);
  if (nseq > INT32_MAX || max_len > INT32_MAX - 1024 || nseq * rows * cols > INT32_MAX) return DUO_ERR_UNSUPPORTED;
  if (nseq == 0) return DUO_OK;
  if (!Q || !O || !lens || (max_len > 0 && !table)) return DUO_ERR_INVALID_ARG;
  if (ldq % 8 || !aligned16(Q)) return DUO_ERR_UNSUPPORTED;
  const size_t need = duo_attention_paged_workspace_size(nseq, heads, g.heads, hd, max_len);
  if (need && (!ws || ws_bytes < need || reinterpret_cast<uintptr_t>(ws) % kAlign)) return DUO_ERR_WORKSPACE;
  if (duo_status d = device_ok(); d != DUO_OK) return d;
  const hipStream_t s = (hipStream_t)stream;
  // exp(x scale) = 2^(x cexp); a negative scale turns the queries' signs instead
  // (never 0: the scores of tokens past the end, -inf, have to stay that)
  const float cexp = std::max((float)(std::fabs(scale) * 1.4426950408889634), 1.4e-45f);
  const uint32_t flip = scale < 0.0 ? 0x80008000u : 0u;
  const int vec = ldo % 2 == 0 && reinterpret_cast<uintptr_t>(O) % 4 == 0;
  return kv_by_format(cache, [&](auto fmt, auto dim) -> duo_status {
    constexpr int FMT = decltype(fmt)::value, HD = decltype(dim)::value;
    using P = PagedGeo<FMT, HD>;
    const int64_t wgs = paged_wgs((double)nseq * (double)rows, cdiv(max_len, P::KEYS), 256 * P::WGS);
    const PagedWork w = {lens, (int)nseq, (int)max_len, (int)rows, (int)cdiv(nseq, 64), nseq * rows >= 2 * 256 * P::WGS};
    Task* const tasks = (Task*)ws;
    float* const part = (float*)((uint8_t*)ws + align_up(wgs * sizeof(Task)));
    constexpr bool Q8 = FMT != DUO_KV_BF16;
    const auto kern = Q8 && cols <= 8 ? paged_kernel<FMT, HD, Q8> : paged_kernel<FMT, HD, false>;
    if (duo_status st = set_max_lds((const void*)kern, 4 * P::WAVE); st != DUO_OK) return st;
    hipLaunchKernelGGL(kern, dim3((unsigned)wgs), dim3(256), 4 * P::WAVE, s, (const uint16_t*)Q, ldq, g, table, ldt, w,
                       (int)group, (int)cols, cexp, flip, (uint16_t*)O, ldo, max_len > 0 ? tasks : nullptr, part, vec);
    DUO_LAUNCH_CHECK();
    if (max_len > P::KEYS && wgs > 1) {  // a row of one tile is never split
      hipLaunchKernelGGL(paged_join_kernel<HD>, dim3((unsigned)wgs, (unsigned)cdiv(cols, 2)), dim3(256), 0, s,
                         (const Task*)tasks, (const float*)part, g.heads, (int)group, (int)cols, (uint16_t*)O, ldo, vec);
      DUO_LAUNCH_CHECK();
    }
    return DUO_OK;
  });
}

}  // extern "C"
