// What the kernels of the paged cache share: a call's sequences, and where a token's row lies.
#pragma once

#include "treekv_internal.h"

namespace tkv {

// The cache as kernels are given it.
struct Pages {
  char *k, *v;
  const int32_t* table;
  int32_t* lens;
  float* weights;
  int32_t* positions;
  int pages, bits, width, cap, B, H, Hkv, G;   // 2^bits rows a page; cap = width << bits
};
inline Pages pages_of(const treekv_paged_cache& c) {
  Pages p;
  p.k = (char*)c.k; p.v = (char*)c.v; p.table = c.table; p.lens = c.lens; p.weights = c.weights; p.positions = c.positions;
  p.pages = c.pages; p.bits = __builtin_ctz(c.page_size); p.width = c.table_width; p.cap = c.table_width * c.page_size;
  p.B = c.batch; p.H = c.q_heads; p.Hkv = c.kv_heads; p.G = c.q_heads / c.kv_heads;
  return p;
}

#if defined(__HIPCC__)

// A sequence's rows in the packed ones, [first, first + n), and its tokens; n = 0 where it has none or is refused (!ok).
struct Seq {
  int first, n, len;
  bool ok;
};
__device__ inline Seq load_seq(const Pages& p, const int32_t* starts, int tokens, int longest, int b) {
  const int lo = starts[b], hi = starts[b + 1], len = p.lens[b];
  Seq s;
  s.ok = lo >= 0 && hi >= lo && hi <= tokens && hi - lo <= longest && len >= hi - lo && len <= p.cap;
  s.first = lo;
  s.n = s.ok ? hi - lo : 0;
  s.len = s.ok ? len : 0;
  return s;
}
// Row of head h in a page, counted in rows of the pool.
__device__ inline size_t pool_row(const Pages& p, int page, int h, int slot) {
  return (((size_t)page * p.Hkv + h) << p.bits) + (slot & ((1 << p.bits) - 1));
}
__device__ inline size_t track_row(const Pages& p, int b, int h) { return ((size_t)b * p.Hkv + h) * p.cap; }

#endif

}  // namespace tkv
