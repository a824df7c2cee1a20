// Host side of the C ABI of speculative decoding: argument checks of treekv_tree_attend, treekv_tree_commit,
// treekv_fork and treekv_qkv_prepare.  The kernels are in treekv_tree.hip, treekv_prefill.hip (the replay of the
// evictions), treekv_fork.hip and treekv_qkv.hip.

#include <stdlib.h>

#include "treekv_internal.h"

using tkv::aligned16;
using tkv::fresh;
using tkv::record_hip;

namespace {

bool nodes_ok(const treekv_ctx* ctx, int n) { return n >= 1 && n <= TREEKV_TREE_MAX_NODES && n <= ctx->cfg.max_chunk; }

// Whether state may move from one context to the other: what describes a unit's state must agree.
bool same_state(const treekv_config& a, const treekv_config& b) {
  return a.budget == b.budget && a.q_heads == b.q_heads && a.kv_heads == b.kv_heads && a.head_dim == b.head_dim &&
         a.dtype == b.dtype && a.n_sink == b.n_sink && a.n_recent == b.n_recent && a.softmax_scale == b.softmax_scale &&
         a.flags == b.flags && a.rope_base == b.rope_base;
}

struct Range {
  uintptr_t lo, hi;      // bytes [lo, hi)
};
bool overlap(const Range& a, const Range& b) { return a.lo < b.hi && b.lo < a.hi; }

}  // namespace

extern "C" {

size_t treekv_tree_scratch_bytes(const treekv_ctx* ctx, int n) {
  return ctx && nodes_ok(ctx, n) ? tkv::tree_scratch_bytes(ctx->p, n) : 0;
}

int treekv_tree_attend(treekv_ctx* ctx, const void* q, const void* k, const void* v, const int32_t* parents, int n,
                       float* out, float* lse, void* scratch, size_t scratch_bytes, void* stream) {
  if (!ctx || !q || !k || !v || !parents || !out) return TREEKV_EINVAL;
  if (!nodes_ok(ctx, n)) return TREEKV_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(scratch)) return TREEKV_EINVAL;
  const size_t need = tkv::tree_scratch_bytes(ctx->p, n);
  if (need > 0 && (!scratch || scratch_bytes < need)) return TREEKV_EINVAL;
  if (!ctx->bound) return TREEKV_ENOWS;
  fresh();
  tkv::Tree t = {q, k, v, parents, n, nullptr, nullptr, nullptr, 0};
  return record_hip(ctx, tkv::launch_tree_attend(ctx->p, t, out, lse, scratch, (hipStream_t)stream));
}

int treekv_tree_commit(treekv_ctx* ctx, const void* q, const void* k, const void* v, const int32_t* parents,
                       const float* lse, int n, const int32_t* path, const int32_t* path_len, int max_len,
                       int32_t* retained, int32_t* n_retained, int32_t* evicted, int32_t* status, void* stream) {
  if (!ctx || !q || !k || !v || !parents || !lse || !path || !path_len || !retained) return TREEKV_EINVAL;
  if (!nodes_ok(ctx, n) || max_len < 1 || max_len > n) return TREEKV_EINVAL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v)) return TREEKV_EINVAL;
  if (!ctx->bound) return TREEKV_ENOWS;
  fresh();
  tkv::Tree t = {q, k, v, parents, n, lse, path, path_len, max_len};
  int rc = tkv::launch_tree_colsums(ctx->p, t, status, (hipStream_t)stream);
  if (rc == TREEKV_OK) rc = tkv::launch_tree_replay(ctx->p, t, retained, n_retained, evicted, (hipStream_t)stream);
  return record_hip(ctx, rc);
}

int treekv_fork(treekv_ctx* ctx, const treekv_ctx* from, const int32_t* src, const int32_t* dst, int count, void* stream) {
  if (!ctx || !from || !src || !dst || count < 1 || count > ctx->cfg.batch) return TREEKV_EINVAL;
  if (!same_state(ctx->cfg, from->cfg)) return TREEKV_EINVAL;
  if (!ctx->bound || !from->bound) return TREEKV_ENOWS;
  const bool inside = ctx->p.K == from->p.K;         // one workspace, whether or not it is one handle
  if (inside && ctx->cfg.batch != from->cfg.batch) return TREEKV_EINVAL;
  // which sequences of ctx are written (1), and may not also be read for another one; one that is given itself (2) may
  unsigned char* written = static_cast<unsigned char*>(calloc((size_t)ctx->cfg.batch, 1));
  if (!written) return TREEKV_EINVAL;
  bool ok = true;
  for (int i = 0; i < count && ok; ++i) {
    ok = dst[i] >= 0 && dst[i] < ctx->cfg.batch && src[i] >= -1 && src[i] < from->cfg.batch && !written[dst[i]];
    if (ok) written[dst[i]] = inside && src[i] == dst[i] ? 2 : 1;
  }
  for (int i = 0; i < count && ok; ++i) ok = !(inside && src[i] >= 0 && src[i] != dst[i] && written[src[i]] == 1);
  free(written);
  if (!ok) return TREEKV_EINVAL;
  fresh();
  return record_hip(ctx, tkv::launch_fork(ctx->p, from->p, src, dst, count, (hipStream_t)stream));
}

int treekv_qkv_prepare(const treekv_qkv_args* args, void* stream) {
  if (!args) return TREEKV_EINVAL;
  const treekv_qkv_args& a = *args;
  if (a.tokens < 1 || (a.dtype != TREEKV_BF16 && a.dtype != TREEKV_F32)) return TREEKV_EINVAL;
  if (!a.q_out && !a.k_out && !a.v_out) return TREEKV_EINVAL;
  if (!a.q != !a.q_out || !a.k != !a.k_out || !a.v != !a.v_out) return TREEKV_EINVAL;
  if ((a.q && a.q_heads < 1) || ((a.k || a.v) && a.kv_heads < 1)) return TREEKV_EINVAL;
  if ((a.flags & ~(TREEKV_ROPE_HALVES | TREEKV_ROPE_TO_PLANES)) || a.flags == TREEKV_ROPE_TO_PLANES) return TREEKV_EINVAL;
  if (!a.positions != !a.inv_freq || a.rotary_dim < 0 || a.rotary_dim > a.head_dim) return TREEKV_EINVAL;
  if (a.positions && a.rotary_dim == 0) return TREEKV_EINVAL;
  if ((a.q_weight && !a.q) || (a.k_weight && !a.k)) return TREEKV_EINVAL;
  if ((a.q_weight || a.k_weight) && !(a.eps >= 0.0f)) return TREEKV_EINVAL;
  if (!aligned16(a.q_weight) || !aligned16(a.k_weight)) return TREEKV_EINVAL;
  if (a.head_dim != 64 && a.head_dim != 128) return TREEKV_EUNSUPPORTED;
  if (a.rotary_dim % 16 != 0 || a.q_heads > 65536 || a.kv_heads > 65536) return TREEKV_EUNSUPPORTED;
  const int64_t esz = a.dtype == TREEKV_BF16 ? 2 : 4;
  const void* in[3] = {a.q, a.k, a.v};
  void* out[3] = {a.q_out, a.k_out, a.v_out};
  const int64_t stride[3] = {a.q_stride, a.k_stride, a.v_stride};
  const int64_t row[3] = {(int64_t)a.q_heads * a.head_dim, (int64_t)a.kv_heads * a.head_dim, (int64_t)a.kv_heads * a.head_dim};
  auto range = [](const void* p, int64_t bytes) { return Range{(uintptr_t)p, (uintptr_t)p + (uintptr_t)(p ? bytes : 0)}; };
  Range ri[3], ro[3];
  for (int x = 0; x < 3; ++x) {
    ri[x] = ro[x] = Range{0, 0};
    if (!in[x]) continue;
    if (!aligned16(in[x]) || !aligned16(out[x])) return TREEKV_EINVAL;
    // (one token has no next one)
    if (a.tokens > 1 && (stride[x] < row[x] || stride[x] > ((int64_t)1 << 40) / esz || stride[x] * esz % 16 != 0)) return TREEKV_EINVAL;
    ri[x] = range(in[x], ((a.tokens > 1 ? (a.tokens - 1) * stride[x] : 0) + row[x]) * esz);
    ro[x] = range(out[x], a.tokens * row[x] * esz);
  }
  const Range small[4] = {range(a.q_weight, a.head_dim * esz), range(a.k_weight, a.head_dim * esz),
                          range(a.positions, (int64_t)a.tokens * 4), range(a.inv_freq, (int64_t)a.rotary_dim * 4)};
  for (int x = 0; x < 3; ++x)
    for (int y = 0; y < 3; ++y) {
      if (x < y && overlap(ro[x], ro[y])) return TREEKV_EINVAL;
      const bool in_place = x == y && out[x] == in[x] && (a.tokens == 1 || stride[x] == row[x]);
      if (!in_place && overlap(ro[x], ri[y])) return TREEKV_EINVAL;
    }
  for (int x = 0; x < 3; ++x)
    for (const Range& r : small)
      if (overlap(ro[x], r)) return TREEKV_EINVAL;
  fresh();
  const int rc = tkv::launch_qkv(a, (hipStream_t)stream);
  (void)tkv::take_hip_error();
  return rc;
}

}  // extern "C"
