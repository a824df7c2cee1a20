// Host side of the C ABI of the paged cache and of the verification of drafts: argument checks of treekv_paged_append,
// treekv_paged_attend, treekv_paged_evict and treekv_tree_verify.  The kernels are in treekv_paged.hip, treekv_evict.hip and
// treekv_verify.hip.

#include <math.h>

#include "treekv_internal.h"

using tkv::aligned16;
using tkv::fresh;

namespace {

// A launch has fewer than 2^32 threads: 2^24 workgroups of 256, of 16 tokens (append), 32 rows (attend; fewer rows are one tile of a
// pair) or 128 slots (weights).  (The merge holds its workgroups to that by itself.)
constexpr int64_t MAX_SLOTS = (int64_t)1 << 30, MAX_TOKENS = (int64_t)1 << 27, MAX_ROWS = (int64_t)1 << 28, MAX_WEIGHED = (int64_t)1 << 30;

struct Range {
  uintptr_t lo, hi;      // bytes [lo, hi)
};
bool overlap(const Range& a, const Range& b) { return a.lo < b.hi && b.lo < a.hi; }
Range range(const void* p, uint64_t bytes) { return Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)(p ? bytes : 0)}; }

int esz_of(const treekv_paged_cache& c) { return c.dtype == TREEKV_F32 ? 4 : 2; }

int cache_ok(const treekv_paged_cache* cache) {
  if (!cache) return TREEKV_EINVAL;
  const treekv_paged_cache& c = *cache;
  if (!c.k || !c.v || !c.table || !c.lens || !aligned16(c.k) || !aligned16(c.v) || !aligned16(c.weights) || !c.weights != !c.positions) return TREEKV_EINVAL;
  if (c.dtype != TREEKV_BF16 && c.dtype != TREEKV_F32) return TREEKV_EINVAL;
  if (c.pages < 1 || c.page_size < 1 || c.table_width < 1 || c.batch < 1 || c.kv_heads < 1 || c.q_heads < 1 || c.q_heads % c.kv_heads != 0)
    return TREEKV_EINVAL;
  if (!isfinite(c.softmax_scale * 1.44269504f)) return TREEKV_EINVAL;        // (logits are scaled by it times log2(e); a logit of 0 would be a NaN)
  if (c.head_dim != 64 && c.head_dim != 128) return TREEKV_EUNSUPPORTED;
  if (c.page_size < 16 || c.page_size > 256 || (c.page_size & (c.page_size - 1))) return TREEKV_EUNSUPPORTED;
  if (c.q_heads > 65536 || (int64_t)c.table_width * c.page_size > MAX_SLOTS || (int64_t)c.batch * c.kv_heads > (1 << 20)) return TREEKV_EUNSUPPORTED;
  return TREEKV_OK;
}

// A strided input [tokens, heads, d] and the bytes it spans; nothing of it may lie in what the call writes.
bool rows_ok(const void* p, int64_t stride, int64_t row, int tokens, int esz) {
  if (!p || !aligned16(p)) return false;
  return tokens == 1 || (stride >= row && stride <= ((int64_t)1 << 40) / esz && stride * esz % 16 == 0);
}
Range rows_range(const void* p, int64_t stride, int64_t row, int tokens, int esz) {
  return range(p, (uint64_t)((tokens > 1 ? (tokens - 1) * stride : 0) + row) * esz);
}
struct CacheRanges {
  Range r[6];      // pools and what is kept per token; table and lens
};
CacheRanges cache_ranges(const treekv_paged_cache& c) {
  const uint64_t pool = (uint64_t)c.pages * c.kv_heads * c.page_size * c.head_dim * esz_of(c);
  const uint64_t track = (uint64_t)c.batch * c.kv_heads * c.table_width * c.page_size * 4;
  return {{range(c.k, pool), range(c.v, pool), range(c.weights, track), range(c.positions, track),
           range(c.table, (uint64_t)c.batch * c.table_width * 4), range(c.lens, (uint64_t)c.batch * 4)}};
}
bool apart(const Range* a, int n, const Range* b, int m) {
  for (int i = 0; i < n; ++i)
    for (int j = 0; j < m; ++j)
      if (&a[i] != &b[j] && overlap(a[i], b[j])) return false;
  return true;
}

int attend_ok(const treekv_paged_cache* c, int tokens, int longest, int weigh) {
  const int rc = cache_ok(c);
  if (rc != TREEKV_OK) return rc;
  if (tokens < 1 || longest < 1 || longest > tokens || (weigh && !c->weights)) return TREEKV_EINVAL;
  const int64_t rows = (int64_t)longest * (c->q_heads / c->kv_heads);
  if (tokens > MAX_TOKENS || rows > MAX_ROWS || rows * c->kv_heads * c->batch > MAX_ROWS) return TREEKV_EUNSUPPORTED;
  if (weigh && (int64_t)c->batch * c->kv_heads * c->table_width * c->page_size > MAX_WEIGHED) return TREEKV_EUNSUPPORTED;
  return TREEKV_OK;
}

}  // namespace

extern "C" {

int treekv_paged_append(const treekv_paged_cache* cache, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                        const int32_t* starts, int tokens, const int32_t* positions, int32_t* status, void* stream) {
  const int rc = cache_ok(cache);
  if (rc != TREEKV_OK) return rc;
  const treekv_paged_cache& c = *cache;
  if (tokens < 1 || !starts || !positions != !c.positions) return TREEKV_EINVAL;
  if (tokens > MAX_TOKENS) return TREEKV_EUNSUPPORTED;
  const int64_t row = (int64_t)c.kv_heads * c.head_dim;
  const int esz = esz_of(c);
  if (!rows_ok(k, k_stride, row, tokens, esz) || !rows_ok(v, v_stride, row, tokens, esz)) return TREEKV_EINVAL;
  const CacheRanges cr = cache_ranges(c);
  const Range in[6] = {rows_range(k, k_stride, row, tokens, esz), rows_range(v, v_stride, row, tokens, esz),
                       range(starts, ((uint64_t)c.batch + 1) * 4), range(positions, (uint64_t)tokens * 4), cr.r[4], cr.r[5]};
  const Range st = range(status, (uint64_t)c.batch * 4);
  if (!apart(cr.r, 4, cr.r, 4) || !apart(cr.r, 4, in, 6) || !apart(&st, 1, cr.r, 4) || !apart(&st, 1, in, 6)) return TREEKV_EINVAL;
  fresh();
  const int got = tkv::launch_paged_append(c, k, v, k_stride, v_stride, starts, tokens, positions, status, (hipStream_t)stream);
  (void)tkv::take_hip_error();
  return got;
}

size_t treekv_paged_attend_scratch_bytes(const treekv_paged_cache* cache, int tokens, int longest, int weigh) {
  return attend_ok(cache, tokens, longest, weigh) == TREEKV_OK ? tkv::paged_attend_scratch_bytes(*cache, tokens, longest, weigh) : 0;
}

int treekv_paged_attend(const treekv_paged_cache* cache, const void* q, int64_t q_stride, const int32_t* starts, int tokens,
                        int longest, void* out, float* lse, int weigh, void* scratch, size_t scratch_bytes, int32_t* status,
                        void* stream) {
  const int rc = attend_ok(cache, tokens, longest, weigh);
  if (rc != TREEKV_OK) return rc;
  const treekv_paged_cache& c = *cache;
  const int64_t row = (int64_t)c.q_heads * c.head_dim;
  const int esz = esz_of(c);
  if (!starts || !out || !aligned16(out) || !aligned16(scratch) || !rows_ok(q, q_stride, row, tokens, esz)) return TREEKV_EINVAL;
  const size_t need = tkv::paged_attend_scratch_bytes(c, tokens, longest, weigh);
  if (need > 0 && (!scratch || scratch_bytes < need)) return TREEKV_EINVAL;
  const CacheRanges cr = cache_ranges(c);
  const Range in[2] = {rows_range(q, q_stride, row, tokens, esz), range(starts, ((uint64_t)c.batch + 1) * 4)};
  const Range to[4] = {range(out, (uint64_t)tokens * row * esz), range(lse, (uint64_t)tokens * c.q_heads * 4),
                       range(need ? scratch : nullptr, need), range(status, (uint64_t)c.batch * 4)};
  if (!apart(to, 4, to, 4) || !apart(to, 4, in, 2) || !apart(to, 4, cr.r, 6)) return TREEKV_EINVAL;
  if (weigh && (!apart(&cr.r[2], 1, in, 2) || !apart(&cr.r[2], 1, cr.r, 6))) return TREEKV_EINVAL;
  fresh();
  const int got = tkv::launch_paged_attend(c, q, q_stride, starts, tokens, longest, out, lse, weigh, scratch, status, (hipStream_t)stream);
  (void)tkv::take_hip_error();
  return got;
}

size_t treekv_paged_evict_scratch_bytes(const treekv_paged_cache* cache) {
  return cache_ok(cache) == TREEKV_OK && cache->weights ? tkv::paged_evict_scratch_bytes(*cache) : 0;
}

int treekv_paged_evict(const treekv_paged_cache* cache, int budget, int n_sink, int n_recent, int32_t* lens_out, void* scratch,
                       size_t scratch_bytes, int32_t* status, void* stream) {
  const int rc = cache_ok(cache);
  if (rc != TREEKV_OK) return rc;
  const treekv_paged_cache& c = *cache;
  if (!c.weights || budget < 1 || n_sink < 0 || n_recent < 0 || (int64_t)n_sink + n_recent > budget) return TREEKV_EINVAL;
  const size_t need = tkv::paged_evict_scratch_bytes(c);
  if (!scratch || !aligned16(scratch) || scratch_bytes < need) return TREEKV_EINVAL;
  const CacheRanges cr = cache_ranges(c);
  const uint64_t ints = (uint64_t)c.batch * 4;
  const Range to[3] = {range(scratch, need), range(status, ints), range(lens_out == c.lens ? nullptr : lens_out, ints)};
  if (!apart(to, 3, to, 3) || !apart(to, 3, cr.r, 6) || !apart(cr.r, 6, cr.r, 6)) return TREEKV_EINVAL;
  fresh();
  const int got = tkv::launch_paged_evict(c, budget, n_sink, n_recent, lens_out, scratch, status, (hipStream_t)stream);
  (void)tkv::take_hip_error();
  return got;
}

size_t treekv_tree_verify_scratch_bytes(int batch, int n, int vocab) {
  return batch >= 1 && batch <= 1 << 20 && n >= 1 && n <= TREEKV_TREE_MAX_NODES && vocab >= 1 && vocab <= 1 << 24 ? tkv::verify_scratch_bytes(batch, n, vocab) : 0;
}

int treekv_tree_verify(const treekv_verify_args* args, void* stream) {
  if (!args) return TREEKV_EINVAL;
  const treekv_verify_args& a = *args;
  if (!a.target || !a.tokens || !a.parents || !a.uniforms || !a.path || !a.path_len || !a.next_token) return TREEKV_EINVAL;
  if (!aligned16(a.target) || !aligned16(a.draft) || !aligned16(a.scratch)) return TREEKV_EINVAL;
  if (a.batch < 1 || a.n < 1 || a.n > TREEKV_TREE_MAX_NODES || a.vocab < 1) return TREEKV_EINVAL;
  if (a.dtype != TREEKV_BF16 && a.dtype != TREEKV_F32) return TREEKV_EINVAL;
  if (a.vocab > 1 << 24 || a.batch > 1 << 20) return TREEKV_EUNSUPPORTED;
  const size_t need = tkv::verify_scratch_bytes(a.batch, a.n, a.vocab);
  if (need > 0 && (!a.scratch || a.scratch_bytes < need)) return TREEKV_EINVAL;
  const uint64_t nodes = (uint64_t)a.batch * a.n, rows = (uint64_t)a.batch * (a.n + 1) * a.vocab * (a.dtype == TREEKV_F32 ? 4 : 2);
  const Range in[5] = {range(a.target, rows), range(a.draft, rows), range(a.tokens, nodes * 4), range(a.parents, nodes * 4),
                       range(a.uniforms, (nodes + a.batch) * 4)};
  const Range to[4] = {range(a.path, nodes * 4), range(a.path_len, (uint64_t)a.batch * 4), range(a.next_token, (uint64_t)a.batch * 4),
                       range(need ? a.scratch : nullptr, need)};
  if (!apart(to, 4, to, 4) || !apart(to, 4, in, 5)) return TREEKV_EINVAL;
  fresh();
  const int got = tkv::launch_verify(a, (hipStream_t)stream);
  (void)tkv::take_hip_error();
  return got;
}

}  // extern "C"
