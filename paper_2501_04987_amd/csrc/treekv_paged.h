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
  bool ok, ascends;          // ascends: its own starts do
};
__device__ inline bool ascends(int lo, int hi, int tokens) { return lo >= 0 && hi >= lo && hi <= tokens; }
// By what its own starts and length say.  Where starts ascend from end to end that is all there is to ask; else the sequence may
// begin before the end of an earlier one, which has the rows then (begins_inside, load_seqs).
__device__ inline Seq load_seq(const Pages& p, const int32_t* starts, int tokens, int longest, int b) {
  const int lo = starts[b], hi = starts[b + 1], len = p.lens[b];
  Seq s;
  s.ascends = ascends(lo, hi, tokens);
  s.ok = s.ascends && hi - lo <= longest && len >= hi - lo && len <= p.cap;
  s.first = lo;
  s.n = s.ok ? hi - lo : 0;
  s.len = s.ok ? len : 0;
  return s;
}
// Whether rows of an earlier sequence lie behind row `first`, where b's begin.  By a whole wave, of one b.
__device__ inline bool begins_inside(const int32_t* starts, int tokens, int b, int first) {
  int end = 0;
  for (int c0 = 0; c0 < b; c0 += 64) {
    const int c = c0 + (int)(threadIdx.x & 63), lo = starts[min(c, b)], hi = starts[min(c, b) + 1];
    end = max(end, c < b && ascends(lo, hi, tokens) && hi > lo ? hi : 0);
  }
  return __any(end > first);
}
// Sequences b0 + lane with all that can be asked of them.  By a whole wave, b0 = 0, 64, .. in turn; `end`: of the rows of those before,
// 0 at first.
__device__ inline Seq load_seqs(const Pages& p, const int32_t* starts, int tokens, int longest, int b0, int& end) {
  const int lane = threadIdx.x & 63, b = b0 + lane;
  Seq s = {0, 0, 0, false, true};
  int mine = 0;                                        // where its rows end
  if (b < p.B) {
    s = load_seq(p, starts, tokens, longest, b);
    if (s.ascends && starts[b + 1] > s.first) mine = starts[b + 1];
  }
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) mine = max(mine, __shfl_up(mine, x, 64));       // (a lane without one below gets its own)
  const int before = __shfl_up(mine, 1, 64);
  if (s.n > 0 && s.first < max(lane ? before : 0, end)) s.ok = false, s.n = s.len = 0;
  end = max(end, __builtin_amdgcn_readlane(mine, 63));
  return s;
}
// All sequences' status, by a workgroup of `threads`; `odd`: starts do not ascend.
__device__ inline void write_status(const Pages& p, const int32_t* starts, int tokens, int longest, bool odd, int32_t* status, int threads) {
  if (__builtin_expect(!odd, 1)) {
    for (int b = threadIdx.x; b < p.B; b += threads) status[b] = load_seq(p, starts, tokens, longest, b).ok ? TREEKV_OK : TREEKV_EINVAL;
  } else if (threadIdx.x < 64) {
    int end = 0;
    for (int b0 = 0; b0 < p.B; b0 += 64) {
      const bool ok = load_seqs(p, starts, tokens, longest, b0, end).ok;
      if (b0 + (int)threadIdx.x < p.B) status[b0 + threadIdx.x] = ok ? TREEKV_OK : TREEKV_EINVAL;
    }
  }
}
// Row of head h in a page, counted in rows of the pool.
__device__ inline size_t pool_row(const Pages& p, int page, int h, int slot) {
  return (((size_t)page * p.Hkv + h) << p.bits) + (slot & ((1 << p.bits) - 1));
}
__device__ inline size_t track_row(const Pages& p, int b, int h) { return ((size_t)b * p.Hkv + h) * p.cap; }

#endif

}  // namespace tkv
