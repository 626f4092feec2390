// Layout of the paged key-value cache, shared by the kernels that write, read and
// attend over it.
#pragma once

#include <type_traits>

#include "common.h"

namespace duo {

constexpr int kKvGroup = 32;       // channels per scale
constexpr int kMaxKvHeads = 4096;  // a page within 2^32 bytes

// Bytes of a cached row and of its scales, most of a code, and what is added to it.
template <int FMT>
struct KvFmt;
template <>
struct KvFmt<DUO_KV_BF16> {
  static constexpr int row(int hd) { return 2 * hd; }
  static constexpr int scales(int) { return 0; }
};
template <>
struct KvFmt<DUO_KV_I8> {
  static constexpr int row(int hd) { return hd; }
  static constexpr int scales(int hd) { return 2 * (hd / kKvGroup); }
  static constexpr int most = 127, bias = 128;
};
template <>
struct KvFmt<DUO_KV_I4> {
  static constexpr int row(int hd) { return hd / 2; }
  static constexpr int scales(int hd) { return 2 * (hd / kKvGroup); }
  static constexpr int most = 7, bias = 8;
};

// Rows of fp16 numbers made of codes (2^6 of them), as chunks' attention keeps them in its workspace.
constexpr int kKvMade = DUO_KV_I4 + 1;
template <>
struct KvFmt<kKvMade> {
  static constexpr int row(int hd) { return 2 * hd; }
  static constexpr int scales(int) { return 0; }
};

// Geometry of one cache as the kernels take it: block = bytes of one head's part of
// a page, [K rows][V rows][K scales][V scales] from its start.
struct KvGeo {
  uint8_t* data;
  int64_t pages, block;
  int shift;  // log2 of the page size
  int heads;
};

template <int FMT, int HD>
__device__ __forceinline__ int kv_rows_at(int which, int shift) {
  return which * (KvFmt<FMT>::row(HD) << shift);
}
template <int FMT, int HD>
__device__ __forceinline__ int kv_scales_at(int which, int shift) {
  return (2 * KvFmt<FMT>::row(HD) + which * KvFmt<FMT>::scales(HD)) << shift;
}

// Checks a cache description (DUO_OK, or why not) and fills in its geometry.
duo_status kv_geo(const duo_kv_cache* c, KvGeo* g);

// f(format, head_dim), as integral constants, of a cache that kv_geo has accepted.
template <class F>
duo_status kv_by_format(const duo_kv_cache* c, const F& f) {
  auto with = [&](auto fmt) {
    return c->head_dim == 128 ? f(fmt, std::integral_constant<int, 128>{}) : f(fmt, std::integral_constant<int, 64>{});
  };
  if (c->format == DUO_KV_BF16) return with(std::integral_constant<int, DUO_KV_BF16>{});
  if (c->format == DUO_KV_I8) return with(std::integral_constant<int, DUO_KV_I8>{});
  return with(std::integral_constant<int, DUO_KV_I4>{});
}

// Where the row of slot `slot` begins in the cache, and its scales (which: 0 K, 1 V).
template <int FMT, int HD>
struct KvRow {
  uint8_t *codes, *scales;
  __device__ KvRow(const KvGeo& g, int64_t slot, int h, int which) {
    const uint32_t page = (uint32_t)(slot >> g.shift), row = (uint32_t)slot & ((1u << g.shift) - 1);
    uint8_t* const blk = g.data + h * g.block + (uint64_t)page * (uint32_t)(g.heads * g.block);
    codes = blk + kv_rows_at<FMT, HD>(which, g.shift) + row * KvFmt<FMT>::row(HD);
    scales = blk + kv_scales_at<FMT, HD>(which, g.shift) + row * KvFmt<FMT>::scales(HD);
  }
};

// A group of 32 channels of one token and head has one scale,
//   s = bf16(max |x| / q),  code = rint(x / s),  q = 127 (8 bits) or 7 (4 bits).
// x and s have eight significant bits, so a quotient that is no half integer is at
// least 2^-16 (relative) away from one, and x / s in fp32 rounds to the code of the
// exact quotient, ties included where the division is exact at them.  kv_encode
// forms x (1/s) and corrects it once by its remainder, which is exact at ties.
//
// The codes of a group of 32 channels, eight per thread and four threads in a row, with what
// is added to them (8 bits: in bytes of q.x, q.y; 4 bits: in q.x), and the scale.
template <int FMT>
__device__ __forceinline__ uint2 kv_encode(const u32x4& x, uint16_t* scale) {
  typedef unsigned short u16v2 __attribute__((ext_vector_type(2)));
  u16v2 most2 = {0, 0};
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    u16v2 v;
    const uint32_t a = x[j] & 0x7fff7fffu;
    __builtin_memcpy(&v, &a, 4);
    most2 = __builtin_elementwise_max(most2, v);
  }
  uint32_t mag = most2[0] > most2[1] ? most2[0] : most2[1];
  mag = max(mag, (uint32_t)__shfl_xor((int)mag, 1));
  mag = max(mag, (uint32_t)__shfl_xor((int)mag, 2));
  constexpr int most = KvFmt<FMT>::most, bias = KvFmt<FMT>::bias;
  // max |x| / q is never within 2^-17 of halfway between two bf16 numbers, so the product
  // rounds as the quotient does
  const uint16_t sb = f32_to_bf16_bits(bf16_bits_to_f32((uint16_t)mag) * (1.0f / most));
  const float s = bf16_bits_to_f32(sb);
  const bool some = mag < 0x7f80u && s >= 1.1754943508222875e-38f;
  *scale = some ? sb : mag < 0x7f80u ? 0 : 0x7fc0u;
  const float inv = some ? __builtin_amdgcn_rcpf(s) : 0.f, div = some ? s : 0.f;
  uint32_t code[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float v = some ? __uint_as_float(j & 1 ? x[j >> 1] & 0xffff0000u : x[j >> 1] << 16) : 0.f;
    const float q = v * inv;
    // + 1.5 2^23: the nearest whole number, ties to even, in the low bits; it lies within
    // the codes, as s is at most 2^-8 too small
    code[j] = __float_as_uint(fmaf(fmaf(-q, div, v), inv, q) + (12582912.0f + bias));
  }
  uint2 q = {0, 0};
  if constexpr (FMT == DUO_KV_I8) {
    auto bytes = [&](int j) {
      return __builtin_amdgcn_perm(__builtin_amdgcn_perm(code[j + 3], code[j + 2], 0x0c0c0400u),
                                   __builtin_amdgcn_perm(code[j + 1], code[j], 0x0c0c0400u), 0x05040100u);
    };
    q.x = bytes(0);
    q.y = bytes(4);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) q.x |= (code[j] & 15u) << (4 * j);
  }
  return q;
}

// Attention of chunks (duo_attention_chunk), checked: the part of it that sequences with more
// than `least` rows (new tokens times heads of a group) take, and its workspace.
struct ChunkCall {
  const void* Q;
  void* O;
  int64_t ldq, ldo, total_q, nseq, max_q, max_len, heads, ldt;
  const duo_kv_cache* cache;
  KvGeo geo;
  const int32_t *table, *lens, *cu_q;
  int window, sinks;
  float cexp;
  uint32_t flip;
};
size_t chunk_rows_ws_bytes(int32_t format, int64_t total_q, int64_t nseq, int64_t heads, int64_t kv_heads, int64_t head_dim, int64_t max_len);
duo_status chunk_rows_run(const ChunkCall& c, int64_t least, void* ws, hipStream_t s);

}  // namespace duo
