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

}  // namespace duo
