// Drafted trees of TreeKV for gfx950: the attention of treekv_tree_attend and the column sums of treekv_tree_commit.
//
// attend   o = SoftMax(q K^T * scale) V for the n nodes of every sequence's tree, over the cached rows, the node's
//          ancestors and the node.  The n * G query rows of a unit share its K and V, so they are the rows of one matrix
//          product.  Logits and probabilities are held in fp32; P enters the second product whole: with bf16 storage it
//          is cut into three bf16 parts (8 + 8 + 8 bits, exact), so nothing of it is rounded.
// commit   the probabilities of the accepted nodes, p = exp(q K^T * scale - lse), summed down the rows into the column
//          accumulators of the chunk path, whose replay then evicts.  K is read again (half the bytes of the attention);
//          keeping the attention's probabilities instead would cost n * G floats a slot.  8 sequences of 32 heads into
//          2048 slots, 8 tokens at most: 29.6 us, 4.6 TB/s of keys.
//
// A wave owns blocks of columns (32 cached rows with bf16 storage, 16 with fp32) and takes them from memory straight into
// registers, in the layout the matrix instructions want: no LDS and no barrier in the loop.  Bound by memory: 16 nodes of 32
// heads, batch 8, 2048 slots 47.6 us, 5.75 TB/s of K and V; one sequence of 8 groups of 4 and 26 nodes by latency, 13.8 us.
//   S^T = K Q^T      A operand: lane (r, g) holds 16 bytes of K row r: the row's pieces 4 s + g in step s
//   O^T += V^T P^T   a lane's logits are columns 4 g + i (+ 16) of row r, which is the B operand as it lies.  The A
//                    operand wants those columns of one dimension; the lane loads 16 bytes (8 at head_dim 64) of each of
//                    those rows, that is, its columns of dimensions r * D/16 .. + D/16 - 1, and one byte permutation per
//                    pair of columns makes the operand of each dimension.
// Column order is free (attention does not depend on it): cached columns are slots in slot order, the free one masked, or,
// with positions re-assigned, logical order, so that column j is at position j.  The tree's own columns follow in blocks of
// their own, masked by the ancestors' bits.
//
// Positions re-assigned: keys are turned in the registers (angles from the context's table), the queries once per workgroup
// in LDS; with bf16 storage both are cut into three bf16 parts, and a logit is the six products above 2^-24.

#include "treekv_internal.h"

namespace tkv {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;

constexpr int TR_THREADS = 512, TR_WAVES = TR_THREADS / 64;
constexpr int MAX_NODES = TREEKV_TREE_MAX_NODES, MAX_WORDS = MAX_NODES / 32;
constexpr float REF_NONE = -3.0e38f;               // reference of a row that has seen nothing: below every logit, and finite, so that exp2(-inf - it) = 0
constexpr float LN2 = 0.6931471805599453f, LOG2E = 1.4426950408889634f;

__device__ inline f32x4_t mfma_bf16(const uint4& a, const uint4& b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ inline f32x16_t mfma_wide(const uint4& a, const uint4& b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
// The high halves of two floats' bits, packed: bf16 by truncation, the first in the low half.
__device__ inline unsigned high_halves(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
__device__ inline float top8(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
// Two fp32 values as bf16 parts whose sum they are: 8 + 8 + 8 bits of the 24.
__device__ inline void cut3(float a, float b, unsigned& h, unsigned& m, unsigned& l) {
  const float a1 = a - top8(a), b1 = b - top8(b);
  h = high_halves(a, b);
  m = high_halves(a1, b1);
  l = high_halves(a1 - top8(a1), b1 - top8(b1));
}
__device__ inline float row_max(float v) {          // over the four lanes, 16 apart, of a row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ inline float row_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// The same value, in a form that keeps what is computed from it from being held across a loop.
__device__ inline int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The tree of one sequence, worked out by the whole workgroup: bit j of sm.anc[i] says that node i attends node j; `up` is
// -1 for a node of the tree and -2 for an absent one.  Generations double from round to round.
struct TreeBits {
  unsigned anc[MAX_NODES][MAX_WORDS];
  int up[MAX_NODES];
};
// Up to 64 nodes: the first wave alone, a node to a lane, generations through lane exchanges instead of barriers.
__device__ inline void build_small_tree(TreeBits& sm, const int32_t* parents, int n) {
  const int i = threadIdx.x;
  if (i < 64) {
    const int p = i < n ? parents[i] : -2;
    int up = p >= -1 && p < i ? p : -2;
    unsigned lo = i < 32 ? 1u << i : 0u, hi = i < 32 ? 0u : 1u << (i - 32);
    while (__any(up >= 0)) {
      const int from = up >= 0 ? up : i;
      const unsigned l = __shfl(lo, from, 64), h = __shfl(hi, from, 64);
      const int next = __shfl(up, from, 64);
      if (up >= 0) { lo |= l; hi |= h; up = next; }
    }
    if (i < n) {
      sm.anc[i][0] = lo;
      sm.anc[i][1] = hi;
      sm.up[i] = up;
    }
  }
  __syncthreads();
}
__device__ inline void build_tree(TreeBits& sm, const int32_t* parents, int n) {
  if (n <= 64) return build_small_tree(sm, parents, n);
  const int i = threadIdx.x, words = (n + 31) / 32;
  if (i < n) {
    const int p = parents[i];
    sm.up[i] = p >= -1 && p < i ? p : -2;
#pragma unroll
    for (int w = 0; w < MAX_WORDS; ++w)
      if (w < words) sm.anc[i][w] = w == i / 32 ? 1u << (i & 31) : 0u;
  }
  for (;;) {
    __syncthreads();
    const int up = i < n ? sm.up[i] : -1;
    unsigned bits[MAX_WORDS] = {};
    int next = up;
    if (up >= 0) {
      next = sm.up[up];
#pragma unroll
      for (int w = 0; w < MAX_WORDS; ++w)
        if (w < words) bits[w] = sm.anc[up][w];
    }
    if (!__syncthreads_or(up >= 0)) break;
    if (up >= 0) {
      sm.up[i] = next;
#pragma unroll
      for (int w = 0; w < MAX_WORDS; ++w)
        if (w < words) sm.anc[i][w] |= bits[w];
    }
  }
}
__device__ inline int depth_of(const TreeBits& sm, int i, int n) {
  int d = -1;
  for (int w = 0; w < (n + 31) / 32; ++w) d += __popc(sm.anc[i][w]);
  return d;
}

// What the kernels are given: the parts of the context and the call that they read (the whole of both would not stay in
// scalar registers).
struct Args {
  const void *K, *V;                 // [U][cap][D]
  const int *meta, *E, *R;
  const float2* tab;                 // angles of distances (positions re-assigned)
  const void *q, *k, *v;
  const int32_t* parents;
  float *out, *lse, *scratch;
  int budget, cap, n_sink, n_recent, m, U, H, Hkv, g_bits, n;      // 2^g_bits query heads a KV head; n nodes
  int row_tiles, slices;
  float scale_log2e;
};

// A unit's columns.  Without re-assigned positions cached column c is slot c, the free slot among them (`hole`, masked), so
// that a block's rows are contiguous; with them, column c is the token at position c.
struct Unit {
  int n, columns, hole;              // cached tokens; cached columns; the free slot, or -1 where it lies behind the tokens
  int rhead, j;                      // order arrays' state
  const int *E, *R;
};
template <bool ROPE>
__device__ inline Unit load_unit(const int* meta, const int* E, const int* R, int m, int n_recent, int unit) {
  const int* w = meta + (size_t)unit * META_STRIDE;
  Unit u;
  u.n = __builtin_amdgcn_readfirstlane(w[META_N]);
  const int free_slot = __builtin_amdgcn_readfirstlane(w[META_FREE]);
  u.hole = !ROPE && free_slot < u.n ? free_slot : -1;
  u.columns = u.hole >= 0 ? u.n + 1 : u.n;
  u.rhead = __builtin_amdgcn_readfirstlane(w[META_RHEAD]);
  u.j = __builtin_amdgcn_readfirstlane(w[META_J]);
  u.E = E + (size_t)unit * 2 * m;
  u.R = R + (size_t)unit * max(n_recent, 1);
  return u;
}
// Slot of the token at position c.
__device__ inline int slot_at(const Unit& u, int budget, int n_sink, int m, int n_recent, int c) {
  if (u.n < budget || c < n_sink) return c;
  c -= n_sink;
  if (c < m) return u.E[tree_index(c, u.j)];
  c += u.rhead - m;
  return u.R[c >= n_recent ? c - n_recent : c];
}

// Operands by storage type.  COLS: columns of a block.  Parts: bf16 parts of a turned value.
template <typename T, int D> struct Ops;

template <int D>
struct Ops<uint16_t, D> {
  static constexpr int COLS = 32, KS = D / 32, NCOL = 8, DPL = D / 16;     // NCOL: columns a lane holds; DPL: its dimensions
  struct Keys { uint4 x[2][KS]; };
  struct Values { uint4 x[8]; };                     // head_dim 64: the first half of each
  __device__ static inline int col(int q4, int j) { return (j >> 2) * 16 + q4 * 4 + (j & 3); }
  __device__ static inline void load_k(Keys& k, int bk, const char* base, unsigned row) {
#pragma unroll
    for (int s = 0; s < KS; ++s) k.x[bk][s] = *reinterpret_cast<const uint4*>(base + row + s * 64);
  }
  __device__ static inline void load_v(Values& v, int j, const char* base, unsigned row) {
    if constexpr (D == 128) v.x[j] = *reinterpret_cast<const uint4*>(base + row);
    else {
      const uint2 r = *reinterpret_cast<const uint2*>(base + row);
      v.x[j] = make_uint4(r.x, r.y, 0, 0);
    }
  }
  __device__ static inline void clear_v(Values& v, int j) { v.x[j] = make_uint4(0, 0, 0, 0); }
  __device__ static inline unsigned word(const uint4& r, int w) { return w == 0 ? r.x : w == 1 ? r.y : w == 2 ? r.z : r.w; }
  // the operand of dimension e: its NCOL columns
  __device__ static inline uint4 dim(const Values& v, int e) {
    const unsigned sel = (e & 1) ? 0x07060302u : 0x05040100u;
    return make_uint4(__builtin_amdgcn_perm(word(v.x[1], e >> 1), word(v.x[0], e >> 1), sel),
                      __builtin_amdgcn_perm(word(v.x[3], e >> 1), word(v.x[2], e >> 1), sel),
                      __builtin_amdgcn_perm(word(v.x[5], e >> 1), word(v.x[4], e >> 1), sel),
                      __builtin_amdgcn_perm(word(v.x[7], e >> 1), word(v.x[6], e >> 1), sel));
  }
  static constexpr int QPARTS = 3;                   // of a turned query
  // queries of one block of 16 rows, from memory (ROPE: from LDS, three parts of `part` elements)
  struct Query { uint4 x[KS]; };
  __device__ static inline void load_q(Query& q, const uint16_t* row, int q4) {
#pragma unroll
    for (int s = 0; s < KS; ++s) q.x[s] = *reinterpret_cast<const uint4*>(row + s * 32 + q4 * 8);
  }
  struct Logits { f32x4_t x[2]; };
  __device__ static inline float& at(Logits& s, int j) { return reinterpret_cast<float*>(&s)[j]; }
};

template <int D>
struct Ops<float, D> {
  static constexpr int COLS = 16, KS = D / 16, NCOL = 4, DPL = D / 16;
  struct Keys { float4 x[1][KS]; };
  struct Values { float x[4][DPL]; };
  __device__ static inline int col(int q4, int j) { return q4 * 4 + j; }
  __device__ static inline void load_k(Keys& k, int, const char* base, unsigned row) {
#pragma unroll
    for (int s = 0; s < KS; ++s) k.x[0][s] = *reinterpret_cast<const float4*>(base + row + s * 64);
  }
  __device__ static inline void load_v(Values& v, int j, const char* base, unsigned row) {
#pragma unroll
    for (int e = 0; e < DPL; e += 4) {
      const float4 r = *reinterpret_cast<const float4*>(base + row + e * 4);
      v.x[j][e] = r.x; v.x[j][e + 1] = r.y; v.x[j][e + 2] = r.z; v.x[j][e + 3] = r.w;
    }
  }
  __device__ static inline void clear_v(Values& v, int j) {
#pragma unroll
    for (int e = 0; e < DPL; ++e) v.x[j][e] = 0.f;
  }
  static constexpr int QPARTS = 1;
  struct Query { float4 x[KS]; };
  __device__ static inline void load_q(Query& q, const float* row, int q4) {
#pragma unroll
    for (int s = 0; s < KS; ++s) q.x[s] = *reinterpret_cast<const float4*>(row + s * 16 + q4 * 4);
  }
  struct Logits { f32x4_t x[1]; };
  __device__ static inline float& at(Logits& s, int j) { return reinterpret_cast<float*>(&s)[j]; }
};

// Turned queries in LDS: QPARTS images of `rows` rows of D elements, rows padded against bank conflicts.
template <typename T, int D>
constexpr int q_row_elems() { return D + 16 / (int)sizeof(T); }

// S^T of one block of columns against one block of 16 rows.
template <int D>
__device__ inline void logits(typename Ops<uint16_t, D>::Logits& s, const typename Ops<uint16_t, D>::Keys& k,
                              const typename Ops<uint16_t, D>::Query& q) {
#pragma unroll
  for (int bk = 0; bk < 2; ++bk) {
    s.x[bk] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < D / 32; ++x) s.x[bk] = mfma_bf16(k.x[bk][x], q.x[x], s.x[bk]);
  }
}
template <int D>
__device__ inline void logits(typename Ops<float, D>::Logits& s, const typename Ops<float, D>::Keys& k,
                              const typename Ops<float, D>::Query& q) {
  f32x4_t a = {0.f, 0.f, 0.f, 0.f}, c = a;
#pragma unroll
  for (int x = 0; x < D / 16; ++x) {
    a = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[0][x].x, q.x[x].x, a, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[0][x].y, q.x[x].y, c, 0, 0, 0);
    a = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[0][x].z, q.x[x].z, a, 0, 0, 0);
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(k.x[0][x].w, q.x[x].w, c, 0, 0, 0);
  }
  s.x[0] = a + c;
}

// One 16-byte piece turned: pairs (2i, 2i+1) by the angles at `cs` (the piece's planes, in order).
__device__ inline void turn_piece(const uint4& raw, const float2* cs, float (&y)[8]) {
  const float4 c01 = reinterpret_cast<const float4*>(cs)[0], c23 = reinterpret_cast<const float4*>(cs)[1];
  const float co[4] = {c01.x, c01.z, c23.x, c23.z}, si[4] = {c01.y, c01.w, c23.y, c23.w};
  float x[8];
  Storage<uint16_t>::widen(raw, x);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y[2 * e] = x[2 * e] * co[e] - x[2 * e + 1] * si[e];
    y[2 * e + 1] = x[2 * e] * si[e] + x[2 * e + 1] * co[e];
  }
}
__device__ inline float4 turn_piece(const float4& x, const float2* cs) {
  const float4 c = *reinterpret_cast<const float4*>(cs);
  return make_float4(x.x * c.x - x.y * c.y, x.x * c.y + x.y * c.x, x.z * c.z - x.w * c.w, x.z * c.w + x.w * c.z);
}
__device__ inline void cut_piece(const float (&y)[8], uint4& h, uint4& m, uint4& l) {
  cut3(y[0], y[1], h.x, m.x, l.x);
  cut3(y[2], y[3], h.y, m.y, l.y);
  cut3(y[4], y[5], h.z, m.z, l.z);
  cut3(y[6], y[7], h.w, m.w, l.w);
}

// The same with positions re-assigned, RB blocks of rows at once (turning the keys is the larger part): `pos[bk]` is the
// position of this lane's key row, `qs` its query row of the first block in LDS (16 rows and QPARTS images further for the
// others).
template <int D, int RB>
__device__ inline void turned_logits(typename Ops<uint16_t, D>::Logits (&s)[RB], const typename Ops<uint16_t, D>::Keys& k,
                                     const float2* tab, const int (&pos)[2], const uint16_t* qs, int part, int q4) {
  constexpr int QR = q_row_elems<uint16_t, D>();
#pragma unroll
  for (int bk = 0; bk < 2; ++bk) {
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) s[rb].x[bk] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    const float2* cs = tab + (size_t)pos[bk] * (D / 2) + q4 * 4;
#pragma unroll
    for (int x = 0; x < D / 32; ++x) {
      float y[8];
      uint4 kh, km, kl;
      turn_piece(k.x[bk][x], cs + x * 16, y);
      cut_piece(y, kh, km, kl);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const uint16_t* q = qs + rb * 16 * QR + x * 32 + q4 * 8;
        const uint4 qh = *reinterpret_cast<const uint4*>(q), qm = *reinterpret_cast<const uint4*>(q + part),
                    ql = *reinterpret_cast<const uint4*>(q + 2 * part);
        f32x4_t a = s[rb].x[bk];
        a = mfma_bf16(kl, qh, a);
        a = mfma_bf16(kh, ql, a);
        a = mfma_bf16(km, qm, a);
        a = mfma_bf16(km, qh, a);
        a = mfma_bf16(kh, qm, a);
        s[rb].x[bk] = mfma_bf16(kh, qh, a);
      }
    }
  }
}
template <int D, int RB>
__device__ inline void turned_logits(typename Ops<float, D>::Logits (&s)[RB], const typename Ops<float, D>::Keys& k,
                                     const float2* tab, const int (&pos)[1], const float* qs, int, int q4) {
  constexpr int QR = q_row_elems<float, D>();
  typename Ops<float, D>::Keys y;
#pragma unroll
  for (int x = 0; x < D / 16; ++x) y.x[0][x] = turn_piece(k.x[0][x], tab + (size_t)pos[0] * (D / 2) + x * 8 + q4 * 2);
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    typename Ops<float, D>::Query q;
    Ops<float, D>::load_q(q, qs + rb * 16 * QR, q4);
    logits<D>(s[rb], y, q);
  }
}

// Turned queries of the workgroup's rows into LDS; `row(r)` gives a row's source and position.
template <typename T, int D, class RowFn>
__device__ inline void stage_turned(T* sq, int rows, int part, const float2* tab, RowFn row) {
  constexpr int EPL = Storage<T>::EPL, PIECES = D / EPL, QR = q_row_elems<T, D>();
  for (int x = threadIdx.x; x < rows * PIECES; x += blockDim.x) {
    const int r = x / PIECES, piece = x % PIECES;
    const T* src;
    int pos;
    row(r, src, pos);
    const float2* cs = tab + (size_t)pos * (D / 2) + piece * (EPL / 2);
    T* dst = sq + r * QR + piece * EPL;
    if constexpr (sizeof(T) == 2) {
      float y[8];
      uint4 h, m, l;
      turn_piece(reinterpret_cast<const uint4*>(src)[piece], cs, y);
      cut_piece(y, h, m, l);
      *reinterpret_cast<uint4*>(dst) = h;
      *reinterpret_cast<uint4*>(dst + part) = m;
      *reinterpret_cast<uint4*>(dst + 2 * part) = l;
    } else {
      *reinterpret_cast<float4*>(dst) = turn_piece(reinterpret_cast<const float4*>(src)[piece], cs);
    }
  }
}

// O^T += V^T P^T for one block of rows; the probabilities are used up.
template <int D>
__device__ inline void add_values(f32x4_t (&o)[D / 16], const typename Ops<uint16_t, D>::Values& v,
                                  const typename Ops<uint16_t, D>::Logits& p) {
  uint4 h, m, l;
  cut3(p.x[0][0], p.x[0][1], h.x, m.x, l.x);
  cut3(p.x[0][2], p.x[0][3], h.y, m.y, l.y);
  cut3(p.x[1][0], p.x[1][1], h.z, m.z, l.z);
  cut3(p.x[1][2], p.x[1][3], h.w, m.w, l.w);
#pragma unroll
  for (int e = 0; e < D / 16; ++e) {
    const uint4 a = Ops<uint16_t, D>::dim(v, e);
    o[e] = mfma_bf16(a, l, o[e]);
    o[e] = mfma_bf16(a, m, o[e]);
    o[e] = mfma_bf16(a, h, o[e]);
  }
}
template <int D>
__device__ inline void add_values(f32x4_t (&o)[D / 16], const typename Ops<float, D>::Values& v,
                                  const typename Ops<float, D>::Logits& p) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < D / 16; ++e) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.x[j][e], p.x[0][j], o[e], 0, 0, 0);
}

// Infinities and NaNs among the values of a block of nodes.  A probability of zero times one of them is a NaN, so a node that
// a row does not attend must not bring them in: they are taken out of the operand, and a row that does attend the node gets
// them added as they are, from memory (a cold path, short rather than fast).
// Per 16-bit half (or word): the top bit set where the value is finite.
__device__ inline unsigned finite_halves(unsigned w) { return ((w & 0x7f807f80u) ^ 0x7f807f80u) + 0x7fff7fffu; }
__device__ inline unsigned finite_word(unsigned w) { return ((w & 0x7f800000u) ^ 0x7f800000u) + 0x7fffffffu; }
template <int D>
__device__ inline bool all_finite(const typename Ops<uint16_t, D>::Values& v) {
  unsigned f = 0x80008000u;
#pragma unroll
  for (int j = 0; j < 8; ++j)
#pragma unroll
    for (int w = 0; w < 4; ++w) f &= finite_halves(Ops<uint16_t, D>::word(v.x[j], w));
  return __all(f == 0x80008000u);
}
template <int D>
__device__ inline bool all_finite(const typename Ops<float, D>::Values& v) {
  unsigned f = 0x80000000u;
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < D / 16; ++e) f &= finite_word(__float_as_uint(v.x[j][e]));
  return __all(f == 0x80000000u);
}
__device__ inline unsigned keep_finite(unsigned w) { return w & ((finite_halves(w) >> 15 & 0x00010001u) * 0xffffu); }
template <int D>
__device__ inline void drop_not_finite(typename Ops<uint16_t, D>::Values& v) {
#pragma unroll
  for (int j = 0; j < 8; ++j)
    v.x[j] = make_uint4(keep_finite(v.x[j].x), keep_finite(v.x[j].y), keep_finite(v.x[j].z), keep_finite(v.x[j].w));
}
template <int D>
__device__ inline void drop_not_finite(typename Ops<float, D>::Values& v) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      const unsigned x = __float_as_uint(v.x[j][e]);
      v.x[j][e] = __uint_as_float(x & (unsigned)((int)finite_word(x) >> 31));
    }
}
// `row`: this lane's dimensions (DPL x 4 of them, from 4 * DPL * q4) of the block's first node; `bits`: what its rows attend.
template <typename T, int D, int RB>
__device__ inline void add_not_finite(f32x4_t (&o)[RB][D / 16], const char* row, size_t node_bytes, int nodes, const unsigned (&bits)[RB]) {
  constexpr int EPL = Storage<T>::EPL, N = D / 4;
#pragma unroll 1
  for (int c = 0; c < nodes; ++c, row += node_bytes) {
#pragma unroll
    for (int x = 0; x < N; x += EPL) {
      float y[EPL];
      Storage<T>::widen(*reinterpret_cast<const uint4*>(row + x * sizeof(T)), y);
#pragma unroll
      for (int z = 0; z < EPL; ++z) {
        const unsigned w = __float_as_uint(y[z]);
        const float odd = __uint_as_float(w & ~(unsigned)((int)finite_word(w) >> 31));       // 0 if it is finite
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) o[rb][(x + z) % (D / 16)][(x + z) / (D / 16)] += (bits[rb] >> c & 1) ? odd : 0.f;
      }
    }
  }
}

// Scratch of a call: one partial result per (unit, row tile, slice): [rows][D] sums relative to the row's reference, then
// [rows][2] reference and sum.
struct Shape {
  int rows_per_tile, row_tiles, slices;
};

// The workgroup's rows from LDS to where they go: the PARTS sums of a row ([part][row][D], rows D + 4 apart) and their
// references and sums ([part][row]) added, then the output or, with several slices, the slice's partial result.
template <int D, int PARTS, int ROWS>
__device__ inline void finish_rows(const Args& p, const TreeBits& tree, const float* so, const float2* sm, int unit, int tile, int slice) {
  const int rows = p.n << p.g_bits, kvh = unit % p.Hkv, b = unit / p.Hkv;
  for (int x = threadIdx.x; x < ROWS * (D / 4); x += blockDim.x) {
    const int r = x / (D / 4), c = x % (D / 4) * 4, row = tile * ROWS + r;
    if (row >= rows) break;
    float M = REF_NONE, L = 0.f;
#pragma unroll
    for (int w = 0; w < PARTS; ++w) M = fmaxf(M, sm[w * ROWS + r].x);
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < PARTS; ++w) {
      const float2 ml = sm[w * ROWS + r];
      const float f = fast_exp2(ml.x - M);
      const float4 y = *reinterpret_cast<const float4*>(so + ((size_t)w * ROWS + r) * (D + 4) + c);
      L = fmaf(ml.y, f, L);
      a.x = fmaf(y.x, f, a.x); a.y = fmaf(y.y, f, a.y); a.z = fmaf(y.z, f, a.z); a.w = fmaf(y.w, f, a.w);
    }
    const int i = row >> p.g_bits;
    const bool present = tree.up[i] == -1;
    if (p.slices > 1) {
      float* part = p.scratch + (((size_t)unit * p.row_tiles + tile) * p.slices + slice) * ROWS * (D + 4) + (size_t)r * (D + 4);
      *reinterpret_cast<float4*>(part + c) = a;
      if (c == 0) *reinterpret_cast<float2*>(part + D) = make_float2(M, present ? L : -1.f);   // below 0: the row is absent
    } else {
      const size_t at = ((size_t)b * p.n + i) * p.H + (kvh << p.g_bits) + (row & ((1 << p.g_bits) - 1));
      const float inv = 1.0f / L;
      *reinterpret_cast<float4*>(p.out + at * D + c) =
          present ? make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (c == 0 && p.lse) p.lse[at] = present ? (M + log2f(L)) * LN2 : -INFINITY;
    }
  }
}

// grid: row tiles x slices x units (remapped so that what reads the same rows shares an XCD's L2).  RB: blocks of 16 rows.
template <typename T, int D, int RB, bool ROPE>
__global__ __launch_bounds__(TR_THREADS, 2) void tree_attend_kernel(Args p) {
  using O = Ops<T, D>;
  constexpr int ROWS = RB * 16, DPL = O::DPL, OR = D + 4;        // OR: floats of a row of sums in LDS
  constexpr int BK = O::COLS / 16, ROWB = D * (int)sizeof(T);
  extern __shared__ __attribute__((aligned(16))) float tr_smem[];
  __shared__ TreeBits tree;
  const int items = p.row_tiles * p.slices * p.U, per_xcd = (items + 7) / 8;
  const int item = ((int)blockIdx.x % 8) * per_xcd + (int)blockIdx.x / 8;
  if (item >= items) return;
  const int tile = item % p.row_tiles, slice = item / p.row_tiles % p.slices, unit = item / (p.row_tiles * p.slices);
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = unit % p.Hkv, b = unit / p.Hkv;
  const Unit u = load_unit<ROPE>(p.meta, p.E, p.R, p.m, p.n_recent, unit);
  const int rows = p.n << p.g_bits, g_mask = (1 << p.g_bits) - 1;
  const int cache_blocks = (u.columns + O::COLS - 1) / O::COLS, blocks = cache_blocks + (p.n + O::COLS - 1) / O::COLS;
  const int begin = (int)((long long)blocks * slice / p.slices), end = (int)((long long)blocks * (slice + 1) / p.slices);

  const char* Ku = (const char*)p.K + (size_t)unit * p.cap * ROWB;
  const char* Vu = (const char*)p.V + (size_t)unit * p.cap * ROWB;
  const size_t node_bytes = (size_t)p.Hkv * ROWB;
  const char* Kn = (const char*)p.k + ((size_t)b * p.n * p.Hkv + kvh) * ROWB;
  const char* Vn = (const char*)p.v + ((size_t)b * p.n * p.Hkv + kvh) * ROWB;

  typename O::Keys k;
  typename O::Values v;
  int slot = 0;                                      // ROPE: of column `lane` (mod COLS) of the block to be loaded next
  auto load_slots = [&](int blk) {
    if constexpr (ROPE)
      if (blk < cache_blocks)
        slot = slot_at(u, p.budget, p.n_sink, p.m, p.n_recent, min(blk * O::COLS + (lane & (O::COLS - 1)), u.n - 1));
  };
  // Lane-dependent addresses are worked out anew at each load: kept across the loop they are thirty registers.
  auto load_keys = [&](int blk) __attribute__((always_inline)) {
    const int l = anew(lane), r = l & 15;
    const unsigned piece = (l >> 4) * 16;
    if (blk < cache_blocks) {
      if constexpr (ROPE) {
#pragma unroll
        for (int bk = 0; bk < BK; ++bk)
          O::load_k(k, bk, Ku + (size_t)(unsigned)__shfl(slot, bk * 16 + r, 64) * ROWB, piece);
      } else {
        const char* base = Ku + (size_t)blk * (O::COLS * ROWB);
        const int last = p.cap - 1 - blk * O::COLS;
#pragma unroll
        for (int bk = 0; bk < BK; ++bk) O::load_k(k, bk, base, (unsigned)min(bk * 16 + r, last) * ROWB + piece);
      }
    } else {
      const int c0 = (blk - cache_blocks) * O::COLS;
#pragma unroll
      for (int bk = 0; bk < BK; ++bk) O::load_k(k, bk, Kn + min(c0 + bk * 16 + r, p.n - 1) * node_bytes, piece);
    }
  };
  auto load_values = [&](int blk) __attribute__((always_inline)) {
    const int l = anew(lane), g = l >> 4;
    const unsigned piece = (l & 15) * (DPL * (int)sizeof(T));
    if (blk < cache_blocks) {
      if constexpr (ROPE) {
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j)
          O::load_v(v, j, Vu + (size_t)(unsigned)__shfl(slot, O::col(g, j), 64) * ROWB, piece);
      } else {
        const char* base = Vu + (size_t)blk * (O::COLS * ROWB);
        const int last = p.cap - 1 - blk * O::COLS;
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j) O::load_v(v, j, base, (unsigned)min(O::col(g, j), last) * ROWB + piece);
      }
    } else {
      const int c0 = (blk - cache_blocks) * O::COLS;
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) O::load_v(v, j, Vn + min(c0 + O::col(g, j), p.n - 1) * node_bytes, piece);
    }
  };
  load_slots(begin + wave);
  if (begin + wave < end) {
    load_keys(begin + wave);
    load_values(begin + wave);
  }
  load_slots(begin + wave + TR_WAVES);

  build_tree(tree, p.parents + (size_t)b * p.n, p.n);

  // this lane's rows (clamped: rows behind the last repeat it and are not written)
  int node[RB];
  constexpr int QR = q_row_elems<T, D>(), Q_PART = ROWS * QR;
  typename O::Query q[RB];
  T* sq = reinterpret_cast<T*>(tr_smem);
  auto query_row = [&](int r) {
    return (const T*)p.q + (((size_t)b * p.n + (r >> p.g_bits)) * p.H + (kvh << p.g_bits) + (r & g_mask)) * D;
  };
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = min(tile * ROWS + rb * 16 + lr, rows - 1);
    node[rb] = r >> p.g_bits;
    if constexpr (!ROPE) O::load_q(q[rb], query_row(r), q4);
  }
  if constexpr (ROPE) {
    stage_turned<T, D>(sq, ROWS, Q_PART, p.tab, [&](int r, const T*& src, int& pos) {
      r = min(tile * ROWS + r, rows - 1);
      src = query_row(r);
      pos = u.n + depth_of(tree, r >> p.g_bits, p.n);
    });
    __syncthreads();
  }

  f32x4_t o[RB][DPL];
  float ref[RB], sum[RB];
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    ref[rb] = REF_NONE;
    sum[rb] = 0.f;
#pragma unroll
    for (int e = 0; e < DPL; ++e) o[rb][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
  }
  const float sc = p.scale_log2e;

  // One block from its operands; the next block's go where its own were as soon as they are used up.  (A second set of
  // operands, requested a whole block ahead, was no faster: head_dim 64 23.4 us with it, 23.9 without at 256 units x 2048 slots;
  // at head_dim 128 it does not fit the registers, 55.4 and 48.7.)
  for (int blk = begin + wave; blk < end; blk += TR_WAVES) {
    const bool cached = blk < cache_blocks;
    const int col0 = (cached ? blk : blk - cache_blocks) * O::COLS, next = blk + TR_WAVES;
    typename O::Logits s[RB];
    if constexpr (ROPE) {
      int pos[BK];
#pragma unroll
      for (int bk = 0; bk < BK; ++bk) {
        const int c = col0 + bk * 16 + lr;
        pos[bk] = cached ? min(c, u.n - 1) : u.n + depth_of(tree, min(c, p.n - 1), p.n);
      }
      turned_logits<D, RB>(s, k, p.tab, pos, sq + lr * QR, Q_PART, q4);
    } else {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) logits<D>(s[rb], k, q[rb]);
    }
    // (scaled once, so that the largest meets a reference of its own bits, however large it is)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) O::at(s[rb], j) *= sc;
    if (next < end) load_keys(next);
    // what a row does not attend
    if (cached) {
      if (col0 + O::COLS > u.columns || (u.hole >= col0 && u.hole < col0 + O::COLS)) {
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j) {
          const int c = col0 + O::col(q4, j);
          if (c >= u.columns || c == u.hole) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) O::at(s[rb], j) = -INFINITY;
            O::clear_v(v, j);                        // whatever the row holds
          }
        }
      }
    } else {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        const unsigned bits = tree.anc[node[rb]][col0 >> 5] >> (col0 & 31);
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j)
          if (!(bits >> O::col(q4, j) & 1)) O::at(s[rb], j) = -INFINITY;
      }
    }
    // The reference need not be the maximum: it is raised when a row's sum passes 2^16 (or overflows, as at first), so the
    // common path has no maxima and no rescaling.
    float fresh_sum[RB];
    typename O::Logits e[RB];
    float worst = 0.f;
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      fresh_sum[rb] = sum[rb];
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) {
        O::at(e[rb], j) = fast_exp2(O::at(s[rb], j) - ref[rb]);
        fresh_sum[rb] += O::at(e[rb], j);
      }
      worst = fmaxf(worst, fresh_sum[rb]);
    }
    if (__any(worst > 0x1p16f)) {
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        float top = O::at(s[rb], 0);
#pragma unroll
        for (int j = 1; j < O::NCOL; ++j) top = fmaxf(top, O::at(s[rb], j));
        const float raised = row_max(fmaxf(ref[rb], top)), by = fast_exp2(ref[rb] - raised);
        fresh_sum[rb] = sum[rb] * by;
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j) {
          O::at(e[rb], j) = fast_exp2(O::at(s[rb], j) - raised);
          fresh_sum[rb] += O::at(e[rb], j);
        }
#pragma unroll
        for (int d = 0; d < DPL; ++d) o[rb][d] *= by;
        ref[rb] = raised;
      }
    }
    if (!cached && !all_finite<D>(v)) {              // (after the raise, which would make a NaN of an infinity)
      unsigned bits[RB];
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) bits[rb] = tree.anc[node[rb]][col0 >> 5] >> (col0 & 31);
      add_not_finite<T, D, RB>(o, Vn + col0 * node_bytes + q4 * (ROWB / 4), node_bytes, min(O::COLS, p.n - col0), bits);
      drop_not_finite<D>(v);
    }
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      sum[rb] = fresh_sum[rb];
      add_values<D>(o[rb], v, e[rb]);
    }
    if (next < end) load_values(next);
    load_slots(next + TR_WAVES);
  }

  // ---- the waves' sums added ----
  float* so = tr_smem;
  float2* sm = reinterpret_cast<float2*>(tr_smem + TR_WAVES * ROWS * OR);
  __syncthreads();                                   // the queries' LDS is free
#pragma unroll
  for (int rb = 0; rb < RB; ++rb) {
    const int r = wave * ROWS + rb * 16 + lr;
    const float l = row_sum(sum[rb]);
    if (q4 == 0) sm[r] = make_float2(ref[rb], l);
    float* dst = so + (size_t)r * OR + q4 * 4 * DPL;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < DPL; e += 4)
        *reinterpret_cast<float4*>(dst + i * DPL + e) = make_float4(o[rb][e][i], o[rb][e + 1][i], o[rb][e + 2][i], o[rb][e + 3][i]);
  }
  __syncthreads();
  finish_rows<D, TR_WAVES, ROWS>(p, tree, so, sm, unit, tile, slice);
}

// A barrier for what the workgroup exchanges through LDS: __syncthreads() also waits for every load on its way to a register.
__device__ inline void lds_barrier() {
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// ---- pieces of the two kernels below, whose waves hold O^T as 32 x 32 blocks: a lane has 16 dimensions, 8 d + 4 (lane / 32)
// + 0 .. 3 of each block, of one row ----
typedef short short4_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) short4_t lds_short4_t;

// O^T += V^T P^T of 32 columns: `p` holds the row's probabilities of columns 8 (i / 4) + 4 (lane / 32) + i % 4, `vp` the lane's
// place in the staged rows (16 lanes fetch 4 rows x 16 dimensions and each gets one dimension's column of them).
template <int D>
__device__ inline void add_wide_values(f32x16_t (&o)[D / 32], const f32x16_t& p, const uint16_t* vp, int v_piece, int v_swz) {
#pragma unroll
  for (int ks = 0; ks < 2; ++ks) {                   // 16 columns: elements 8 ks .. + 7
    uint4 h, m, l;
    cut3(p[ks * 8], p[ks * 8 + 1], h.x, m.x, l.x);
    cut3(p[ks * 8 + 2], p[ks * 8 + 3], h.y, m.y, l.y);
    cut3(p[ks * 8 + 4], p[ks * 8 + 5], h.z, m.z, l.z);
    cut3(p[ks * 8 + 6], p[ks * 8 + 7], h.w, m.w, l.w);
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      uint2 a[2];
#pragma unroll
      for (int x = 0; x < 2; ++x)                    // (multiples of 8 rows: a row's swizzle is that of its last three bits)
        a[x] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                   (lds_short4_t*)(vp + (ks * 16 + x * 8) * D + ((d * 4 + v_piece) ^ v_swz) * 8)));
      const uint4 v = make_uint4(a[0].x, a[0].y, a[1].x, a[1].y);
      o[d] = mfma_wide(v, l, o[d]);
      o[d] = mfma_wide(v, m, o[d]);
      o[d] = mfma_wide(v, h, o[d]);
    }
  }
}
// Rows of a staged tile of V that must not reach the product whatever they hold, cleared by the whole workgroup: of cached
// columns the free slot's and those behind the last token, of nodes the infinities and NaNs (true: there were some).
template <int D>
__device__ inline void clear_cached(uint16_t* vp, int c0, int columns, int hole) {
  for (int x = threadIdx.x; x < 64 * (D / 8); x += blockDim.x) {
    const int c = c0 + x / (D / 8);
    if (c >= columns || c == hole) reinterpret_cast<uint4*>(vp)[x] = make_uint4(0, 0, 0, 0);
  }
}
template <int D>
__device__ inline bool clear_odd(uint16_t* vp) {
  bool odd = false;
  for (int x = threadIdx.x; x < 64 * (D / 8); x += blockDim.x) {
    const uint4 was = reinterpret_cast<uint4*>(vp)[x];
    const uint4 w = make_uint4(keep_finite(was.x), keep_finite(was.y), keep_finite(was.z), keep_finite(was.w));
    if (w.x != was.x || w.y != was.y || w.z != was.z || w.w != was.w) {
      odd = true;
      reinterpret_cast<uint4*>(vp)[x] = w;
    }
  }
  return __syncthreads_or(odd);
}
// The nodes' infinities and NaNs, from memory, to a row that attends them (`row_v`: this lane's first dimension of the first).
template <int DB>
__device__ inline void add_odd_values(f32x16_t (&o)[DB], const char* row_v, size_t node_bytes, int nodes, unsigned bits) {
#pragma unroll 1
  for (int c = 0; c < nodes; ++c, row_v += node_bytes) {
#pragma unroll
    for (int d = 0; d < DB * 4; ++d) {
      const uint2 w = *reinterpret_cast<const uint2*>(row_v + d * 16);
      const unsigned x[4] = {w.x << 16, w.x & 0xffff0000u, w.y << 16, w.y & 0xffff0000u};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float y = __uint_as_float(x[i] & ~(unsigned)((int)finite_word(x[i]) >> 31));       // 0 if it is finite
        o[d >> 2][(d & 3) * 4 + i] += (bits >> c & 1) ? y : 0.f;
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0f70);                // (no wait of the compiler's for these in the caller's loop)
}
template <int D>
__device__ inline void leave_wide_sums(const f32x16_t (&o)[D / 32], float ref, float sum, float* so, float2* sm, int r, int hi) {
  sum += __shfl_xor(sum, 32, 64);
  if (hi == 0) sm[r] = make_float2(ref, sum);
#pragma unroll
  for (int d = 0; d < D / 8; ++d)
    *reinterpret_cast<float4*>(so + (size_t)r * (D + 4) + d * 8 + hi * 4) =
        make_float4(o[d >> 2][(d & 3) * 4], o[d >> 2][(d & 3) * 4 + 1], o[d >> 2][(d & 3) * 4 + 2], o[d >> 2][(d & 3) * 4 + 3]);
}

// ---------------------------------------------------------------------------------------------
// attend, many rows: bf16 storage, tiles of columns shared by the workgroup's waves
// ---------------------------------------------------------------------------------------------
// The kernel above reads every row of K and V once per 32 rows.  Here a workgroup owns 128 rows: RG groups of 32 x two waves
// that take one half of a tile's 64 columns each.  64 nodes of 8 groups of 4, batch 16, 4096 slots: 145-158 us (from card to
// card), 0.47-0.43 PFLOP/s of the formula's operations and, P being three parts, twice that of matrix instructions.  The matrix
// unit is busy for 53 us of it and the vector unit for some 50, mostly one after the other: both waves of a SIMD pass the same barrier
// every tile and so are in the same phase of it.  Tiles come by asynchronous copies into LDS, row-major as they lie in memory
// with the 16-byte pieces of a row swizzled, so that the operand reads (16 bytes of a row for K, the transposing read for V)
// spread over the banks.  v_mfma_f32_32x32x16_bf16: a wave's vector instructions issue beside it, while a 16x16x32 holds them up
// (256 rows into 4096 slots 149 us with those, 145 with these).  A lane then holds 16 columns of one row.
// Iteration t forms the logits of tile t + 1 (matrix unit) beside the probabilities of tile t (vector unit) and ends with tile
// t's product with V.  Four stages: tile t + 1 has landed, t + 2 and t + 3 are on their way, and the stage that t + 3 goes to
// was last read in iteration t - 1, before the barrier.
constexpr int TILE_COLS = 64, STAGES = 4;

// async_copy16 with the source as a wave-uniform base and a lane's byte offset.
__device__ inline void async_copy16_at(const char* uniform_base, unsigned lane_offset, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :: "v"(lane_offset), "s"(uniform_base), "s"(lds_base) : "memory");
}

template <int D>
__global__ __launch_bounds__(TR_THREADS, 2) void tree_attend_tiled_kernel(Args p) {
  constexpr int RG = 4, CG = 2, WAVES = TR_WAVES, THREADS = TR_THREADS;
  constexpr int ROWS = RG * 32, KS = D / 16, DB = D / 32, OR = D + 4, ROWB = D * 2;
  constexpr int PARTS = D / 8, RPC = 64 / PARTS;                   // 16-byte pieces of a row, rows of a 1 KB copy
  constexpr int WROWS = TILE_COLS / WAVES, CPW = WROWS / RPC;   // tile rows a wave copies, its copies of K (and of V) a tile
  constexpr int TILE = TILE_COLS * D;                              // elements of a staged tile
  static_assert(RG * CG == WAVES && TILE_COLS == CG * 32, "a wave takes 32 columns of every tile");
  extern __shared__ __attribute__((aligned(1024))) float tr_smem[];
  __shared__ TreeBits tree;
  uint16_t* k_stages = reinterpret_cast<uint16_t*>(tr_smem);
  uint16_t* v_stages = k_stages + STAGES * TILE;
  auto kswz = [](int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); };
  auto vswz = [](int r) { return D == 128 ? ((r & 7) << 1) : (((r >> 1) & 3) << 1); };
  const int items = p.row_tiles * p.slices * p.U, per_xcd = (items + 7) / 8;
  const int item = ((int)blockIdx.x % 8) * per_xcd + (int)blockIdx.x / 8;
  if (item >= items) return;
  const int tile = item % p.row_tiles, slice = item / p.row_tiles % p.slices, unit = item / (p.row_tiles * p.slices);
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), rg = wave / CG, cg = wave % CG;
  const int kvh = unit % p.Hkv, b = unit / p.Hkv;
  const Unit u = load_unit<false>(p.meta, p.E, p.R, p.m, p.n_recent, unit);
  const int rows = p.n << p.g_bits, g_mask = (1 << p.g_bits) - 1, row = min(tile * ROWS + rg * 32 + lr, rows - 1);
  const int cache_tiles = (u.columns + TILE_COLS - 1) / TILE_COLS, tiles = cache_tiles + (p.n + TILE_COLS - 1) / TILE_COLS;
  const int begin = (int)((long long)tiles * slice / p.slices), end = (int)((long long)tiles * (slice + 1) / p.slices);

  const char* Ku = (const char*)p.K + (size_t)unit * p.cap * ROWB;
  const char* Vu = (const char*)p.V + (size_t)unit * p.cap * ROWB;
  const size_t node_bytes = (size_t)p.Hkv * ROWB;
  const char* Kn = (const char*)p.k + ((size_t)b * p.n * p.Hkv + kvh) * ROWB;
  const char* Vn = (const char*)p.v + ((size_t)b * p.n * p.Hkv + kvh) * ROWB;

  // copy x of wave w fills tile rows w * WROWS + x * RPC + lane / PARTS; a lane takes the piece whose place its own is
  const unsigned lds_wave = __builtin_amdgcn_readfirstlane(lds_address(k_stages)) + wave * CPW * 1024;
  const int a_row = wave * WROWS + lane / PARTS, a_slot = lane % PARTS;
  auto request = [=](int t) {
    const unsigned m0 = lds_wave + ((t - begin) & (STAGES - 1)) * (TILE * 2), vm0 = m0 + STAGES * (TILE * 2);
    if (t < cache_tiles) {
      const char* kb = Ku + (size_t)t * (TILE_COLS * ROWB);
      const char* vb = Vu + (size_t)t * (TILE_COLS * ROWB);
      const int last = p.cap - 1 - t * TILE_COLS;                  // rows behind the last slot repeat it
#pragma unroll
      for (int x = 0; x < CPW; ++x) {
        const int r = a_row + x * RPC;
        const unsigned row = (unsigned)min(r, last) * ROWB;
        async_copy16_at(kb, row + (a_slot ^ kswz(r)) * 16, m0 + x * 1024);
        async_copy16_at(vb, row + (a_slot ^ vswz(r)) * 16, vm0 + x * 1024);
      }
    } else {
      const int c0 = (t - cache_tiles) * TILE_COLS;
#pragma unroll
      for (int x = 0; x < CPW; ++x) {
        const int r = a_row + x * RPC;
        const size_t row = min(c0 + r, p.n - 1) * node_bytes;
        async_copy16(Kn + row + (a_slot ^ kswz(r)) * 16, m0 + x * 1024);
        async_copy16(Vn + row + (a_slot ^ vswz(r)) * 16, vm0 + x * 1024);
      }
    }
  };
#pragma unroll
  for (int x = 0; x < STAGES - 1; ++x)
    if (begin + x < end) request(begin + x);

  // this lane's row (clamped: rows behind the last repeat it and are not written)
  const int node = row >> p.g_bits;
  uint4 q[KS];
  {
    const uint16_t* src = (const uint16_t*)p.q + (((size_t)b * p.n + node) * p.H + (kvh << p.g_bits) + (row & g_mask)) * D + hi * 8;
#pragma unroll
    for (int x = 0; x < KS; ++x) q[x] = *reinterpret_cast<const uint4*>(src + x * 16);
  }
  build_tree(tree, p.parents + (size_t)b * p.n, p.n);

  f32x16_t o[DB];
  float ref = REF_NONE, sum = 0.f;
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x16_t{};
  // Logits are scaled as the reference is taken from them, in one step. Past 2^20 the rounding of the reference alone could
  // carry an exponential past the largest number (from 2^31 on): such a row's logits are scaled first (factor = 1). Scaling all of
  // them first costs 3 us of 150 (64 nodes of 32 heads in 8 groups, batch 16, 4096 slots).
  const float sc = p.scale_log2e;
  float factor = sc;
  bool any_large = false;                            // in some row of the wave
  // where this lane reads its wave's operands from, inside a stage: K row lr; for V, 16 lanes fetch 4 rows x 16 dimensions
  // and each gets one dimension's column of them
  const int l16 = lane & 15, v_row = hi * 4 + (l16 >> 2);
  const int k_swz = kswz(lr), k_off = (cg * 32 + lr) * D, v_off = (cg * 32 + v_row) * D + (lane & 1) * 4;
  const int v_piece = ((lane >> 4) & 1) * 2 + ((l16 >> 1) & 1);

  // S^T of this wave's columns of tile t
  auto form_logits = [&](int t, f32x16_t& s) __attribute__((always_inline)) {
    const uint16_t* kp = k_stages + ((t - begin) & (STAGES - 1)) * TILE + k_off;
    s = f32x16_t{};
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const uint4 k = *reinterpret_cast<const uint4*>(kp + ((x * 2 + hi) ^ k_swz) * 8);
      s = mfma_wide(k, q[x], s);
    }
  };
  // column, inside the wave's 32, of element i
  auto col_of = [&](int i) { return (i >> 2) * 8 + hi * 4 + (i & 3); };
  auto clear_rows = [&](int t) -> bool {             // in a tile that has landed
    uint16_t* vp = v_stages + ((t - begin) & (STAGES - 1)) * TILE;
    if (t >= cache_tiles) return clear_odd<D>(vp);
    const int c0 = t * TILE_COLS;
    if (c0 + TILE_COLS > u.columns || (u.hole >= c0 && u.hole < c0 + TILE_COLS)) clear_cached<D>(vp, c0, u.columns, u.hole);
    return false;
  };

  // The queries have arrived, in a form the compiler sees: it does not know of the copies above, and a wait of its own for
  // them inside the loop would wait for the tiles on their way.
  __builtin_amdgcn_s_waitcnt(0x0f70);                // vmcnt(0)
  __syncthreads();
  bool odd = begin < end && clear_rows(begin);       // of tile t
  f32x16_t s = {};
  if (begin < end) form_logits(begin, s);
  __syncthreads();
  for (int t = begin; t < end; ++t) {
    bool odd_next = false;
    if (t > begin) {                                 // tile t + 1 has landed for every wave, and tile t - 1 is done with
      if (t + 2 < end) wait_vmcnt<2 * CPW>(); else wait_vmcnt<0>();
      __syncthreads();
    }
    if (t + 3 < end) request(t + 3);
    if (t + 1 < end) odd_next = clear_rows(t + 1);
    // what a row does not attend
    const bool cached = t < cache_tiles;
    const int col0 = (cached ? t : t - cache_tiles) * TILE_COLS + cg * 32;
    if (__builtin_expect(any_large, 0)) {
      const float first = factor != sc ? sc : 1.0f;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] *= first;
    }
    if (cached) {
      if (col0 + 32 > u.columns || (u.hole >= col0 && u.hole < col0 + 32)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const int c = col0 + col_of(i);
          s[i] = c < u.columns && c != u.hole ? s[i] : -INFINITY;
        }
      }
    } else {
      const unsigned bits = (col0 < p.n ? tree.anc[node][col0 >> 5] : 0u) >> (hi * 4);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = (bits >> ((i >> 2) * 8 + (i & 3)) & 1) ? s[i] : -INFINITY;
    }
    // The reference need not be the maximum: it is raised where a logit passes it by 2^8 (as at first), which is rare.
    {
      float top = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
      if (__any(fmaf(top, factor, -ref) > 8.0f)) {
        float raised = fmaxf(ref, top * factor);
        raised = fmaxf(raised, __shfl_xor(raised, 32, 64));
        const float by = fast_exp2(ref - raised);
        sum *= by;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= by;
        ref = raised;
        const bool large = factor == sc && fabsf(ref) > 0x1p20f;
        if (__any(large)) {
          const float first = large ? sc : 1.0f;
#pragma unroll
          for (int i = 0; i < 16; ++i) s[i] *= first;
          if (large) factor = 1.0f;
          any_large = true;
        }
      }
    }
    if (odd && col0 < p.n)                           // (after the raise, which would make a NaN of an infinity)
      add_odd_values<DB>(o, Vn + col0 * node_bytes + hi * 8, node_bytes, min(32, p.n - col0), tree.anc[node][col0 >> 5]);
    // logits of tile t + 1 (behind the last one: of whatever the stage holds, unused); probabilities of tile t and their
    // product with V
    f32x16_t next;
    form_logits(t + 1, next);
    const uint16_t* vp = v_stages + ((t - begin) & (STAGES - 1)) * TILE + v_off;
    float add = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = fast_exp2(fmaf(s[i], factor, -ref));
      add += s[i];
    }
    sum += add;
    add_wide_values<D>(o, s, vp, v_piece, vswz(v_row));
    s = next;
    odd = odd_next;
  }
  __syncthreads();

  float* so = tr_smem;                               // [CG][ROWS][D + 4]
  float2* sm = reinterpret_cast<float2*>(tr_smem + CG * ROWS * OR);
  leave_wide_sums<D>(o, ref, sum, so, sm, cg * ROWS + rg * 32 + lr, hi);
  __syncthreads();
  finish_rows<D, CG, ROWS>(p, tree, so, sm, unit, tile, slice);
}

// ---------------------------------------------------------------------------------------------
// attend, positions re-assigned: bf16 storage, keys turned once for 64 rows
// ---------------------------------------------------------------------------------------------
// Turning a key and cutting it costs more than its products with 32 queries, so here the four waves of a workgroup (two groups
// of 32 rows x two halves of a tile's 64 columns) share the work: a thread turns a quarter of one row, cuts it and leaves the
// parts in LDS, with V as it is.  Turned values are cut in two fp16 parts (11 + 11 bits, rounded: what is left is 2^-24 of the
// value), which takes three products (what is left out, low times low, is 2^-24 of the product) where bf16 parts take six; a
// row is scaled by a power of two so that its largest element is near 2^13, and the scales go back on with the softmax's.
// The next tile is on its way while one is worked on, keys and angles to registers, V to the other of its two stages; two
// workgroups share a compute unit and fill each other's waits at the two barriers of a tile.  13 nodes of 8 groups of 4, batch
// 8, 2048 slots: 42.5 us with the merge, of which some 15 do not grow with the cache (order arrays, first angles, the queries'
// cut, partial results); a tile more costs 6 us on every unit.  The vector unit is busy for some 14 us of it, the matrix unit for 5.
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8_t;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2_t;
constexpr int TURN_THREADS = 256, TURN_ROWS = 64;

__device__ inline f32x16_t mfma_half(const uint4& a, const uint4& b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8_t, a), __builtin_bit_cast(f16x8_t, b), c, 0, 0, 0);
}
// Two values as fp16 parts h + l.
__device__ inline void cut2(float a, float b, unsigned& h, unsigned& l) {
  const f16x2_t hv = {(_Float16)a, (_Float16)b};
  const f16x2_t lv = {(_Float16)(a - (float)hv.x), (_Float16)(b - (float)hv.y)};
  h = __builtin_bit_cast(unsigned, hv);
  l = __builtin_bit_cast(unsigned, lv);
}
// Larger of two packed bf16 magnitudes, half by half (as 15-bit integers).
__device__ inline unsigned max_magnitudes(unsigned a, unsigned b) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(unsigned, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a & 0x7fff7fffu), __builtin_bit_cast(u16x2, b & 0x7fff7fffu)));
}
// The power of two that brings a row's largest magnitude (packed bf16) to [2^13, 2^14), and its inverse.
__device__ inline float row_scale(unsigned packed, float& inverse) {
  const unsigned top = max(packed & 0xffffu, packed >> 16), e = top >> 7;        // biased exponent
  const bool odd = e == 0 || e == 255;                                           // nothing (or next to it), or not finite
  inverse = odd ? 1.f : __uint_as_float(max(e, 14u) - 13 << 23);                 // 2^(e - 127 - 13)
  return odd ? 1.f : __uint_as_float(min(267u - max(e, 14u), 254u) << 23);       // 2^(127 + 13 - e)
}
// One 16-byte piece scaled, turned and cut.
__device__ inline void turn_cut(const uint4& raw, float scale, const float4& c01, const float4& c23, uint4& h, uint4& l) {
  const float co[4] = {c01.x, c01.z, c23.x, c23.z}, si[4] = {c01.y, c01.w, c23.y, c23.w};
  float x[8], y[8];
  Storage<uint16_t>::widen(raw, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] *= scale;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    y[2 * e] = x[2 * e] * co[e] - x[2 * e + 1] * si[e];
    y[2 * e + 1] = x[2 * e] * si[e] + x[2 * e + 1] * co[e];
  }
  cut2(y[0], y[1], h.x, l.x);
  cut2(y[2], y[3], h.y, l.y);
  cut2(y[4], y[5], h.z, l.z);
  cut2(y[6], y[7], h.w, l.w);
}

template <int D>
__global__ __launch_bounds__(TURN_THREADS, 2) void tree_attend_turned_kernel(Args p) {
  constexpr int RG = 2, CG = 2, ROWS = TURN_ROWS, KS = D / 16, DB = D / 32, OR = D + 4, ROWB = D * 2, PARTS = D / 8;
  constexpr int PER = PARTS / 4;                                   // 16-byte pieces of a thread: four threads a row
  constexpr int TILE = TILE_COLS * D;                              // elements of one part of a tile
  static_assert(TILE_COLS * 4 == TURN_THREADS && RG * CG * 64 == TURN_THREADS, "a row to four threads");
  extern __shared__ __attribute__((aligned(1024))) float tr_smem[];
  __shared__ TreeBits tree;
  __shared__ float col_scale[TILE_COLS];
  uint16_t* kh = reinterpret_cast<uint16_t*>(tr_smem);
  uint16_t* kl = kh + TILE;
  uint16_t* vs = kl + TILE;                          // two stages
  auto kswz = [](int r) { return D == 128 ? (r & 15) : ((r >> 1) & 7); };
  auto vswz = [](int r) { return D == 128 ? ((r & 7) << 1) : (((r >> 1) & 3) << 1); };
  const int items = p.row_tiles * p.slices * p.U, per_xcd = (items + 7) / 8;
  const int item = ((int)blockIdx.x % 8) * per_xcd + (int)blockIdx.x / 8;
  if (item >= items) return;
  const int tile = item % p.row_tiles, slice = item / p.row_tiles % p.slices, unit = item / (p.row_tiles * p.slices);
  const int tid = threadIdx.x, lane = tid & 63, lr = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), rg = wave / CG, cg = wave % CG;
  const int kvh = unit % p.Hkv, b = unit / p.Hkv;
  const Unit u = load_unit<true>(p.meta, p.E, p.R, p.m, p.n_recent, unit);
  const int rows = p.n << p.g_bits, g_mask = (1 << p.g_bits) - 1, row = min(tile * ROWS + rg * 32 + lr, rows - 1);
  const int cache_tiles = (u.n + TILE_COLS - 1) / TILE_COLS, tiles = cache_tiles + (p.n + TILE_COLS - 1) / TILE_COLS;
  const int begin = (int)((long long)tiles * slice / p.slices), end = (int)((long long)tiles * (slice + 1) / p.slices);
  const char* Ku = (const char*)p.K + (size_t)unit * p.cap * ROWB;
  const char* Vu = (const char*)p.V + (size_t)unit * p.cap * ROWB;
  const size_t node_bytes = (size_t)p.Hkv * ROWB;
  const char* Kn = (const char*)p.k + ((size_t)b * p.n * p.Hkv + kvh) * ROWB;
  const char* Vn = (const char*)p.v + ((size_t)b * p.n * p.Hkv + kvh) * ROWB;

  // this thread's part of a tile of keys: row t_row, pieces 4 x + l % 4 (four lanes take 64 bytes of a row at once).  Its wave
  // copies the same 16 rows of V: copy x fills tile rows 16 wave + x * RPC + lane / PARTS, a lane taking the piece whose place
  // its own is.
  constexpr int RPC = 64 / PARTS, CPW = 16 / RPC;
  const int t_row = tid >> 2;
  uint4 raw_k[PER];
  float4 angles[2 * PER];
  const unsigned lds_v = __builtin_amdgcn_readfirstlane(lds_address(vs)) + wave * CPW * 1024;
  int slot = 0;                                      // of its row in the tile to be requested next
  auto find_slot = [&](int t) {
    if (t < cache_tiles) slot = slot_at(u, p.budget, p.n_sink, p.m, p.n_recent, min(t * TILE_COLS + t_row, u.n - 1));
  };
  // V first: what waits for the keys then waits for it too
  auto request = [&](int t) {
    const bool cached = t < cache_tiles;
    const int c0 = (cached ? t : t - cache_tiles) * TILE_COLS;
    const unsigned m0 = lds_v + ((t - begin) & 1) * (TILE * 2);
    const int l = anew(lane), t_row = wave * 16 + (l >> 2), quarter = l & 3;
#pragma unroll
    for (int x = 0; x < CPW; ++x) {
      const int r = x * RPC + l / PARTS, piece = (l % PARTS) ^ vswz(r);       // (16 rows a wave: its first row's swizzle is 0)
      const size_t at = cached ? (size_t)(unsigned)__shfl(slot, r * 4, 64) * ROWB : min(c0 + wave * 16 + r, p.n - 1) * node_bytes;
      async_copy16((cached ? Vu : Vn) + at + piece * 16, m0 + x * 1024);
    }
    const int node = min(c0 + t_row, p.n - 1);
    int pos = min(c0 + t_row, u.n - 1);
    if (!cached) pos = u.n + depth_of(tree, node, p.n);
    const uint4* kr = reinterpret_cast<const uint4*>(cached ? Ku + (size_t)(unsigned)slot * ROWB : Kn + node * node_bytes) + quarter;
    const float4* cs = reinterpret_cast<const float4*>(p.tab + (size_t)pos * (D / 2)) + quarter * 2;
#pragma unroll
    for (int x = 0; x < PER; ++x) raw_k[x] = kr[x * 4];
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      angles[2 * x] = cs[x * 8];
      angles[2 * x + 1] = cs[x * 8 + 1];
    }
  };
  // its part of the keys into LDS
  auto put = [&]() {
    const int l = anew(lane), t_row = wave * 16 + (l >> 2), quarter = l & 3;
    unsigned top = 0;
#pragma unroll
    for (int x = 0; x < PER; ++x)
      top = max_magnitudes(max_magnitudes(max_magnitudes(raw_k[x].x, raw_k[x].y), max_magnitudes(raw_k[x].z, raw_k[x].w)), top);
    top = max_magnitudes(top, __shfl_xor(top, 1, 64));
    top = max_magnitudes(top, __shfl_xor(top, 2, 64));
    float inverse;
    const float scale = row_scale(top, inverse);
    if (quarter == 0) col_scale[t_row] = inverse;
#pragma unroll
    for (int x = 0; x < PER; ++x) {
      uint4 high, low;
      turn_cut(raw_k[x], scale, angles[2 * x], angles[2 * x + 1], high, low);
      const int place = t_row * PARTS + ((x * 4 + quarter) ^ kswz(t_row));
      reinterpret_cast<uint4*>(kh)[place] = high;
      reinterpret_cast<uint4*>(kl)[place] = low;
    }
  };
  // (the first tile and the queries are asked for before the tree is known, where they do not hang on it; a slice without a
  // tile, of which a cache that is still filling has some, asks for nothing: nobody would wait for its copies into LDS, which
  // becomes the sums')
  find_slot(begin);
  if (begin < cache_tiles && begin < end) request(begin);
  const int node = row >> p.g_bits;
  uint4 raw_q[KS];
  {
    const uint4* src = reinterpret_cast<const uint4*>((const uint16_t*)p.q + (((size_t)b * p.n + node) * p.H + (kvh << p.g_bits) + (row & g_mask)) * D);
#pragma unroll
    for (int x = 0; x < KS; ++x) raw_q[x] = src[x * 2 + hi];
  }
  build_tree(tree, p.parents + (size_t)b * p.n, p.n);
  if (begin >= cache_tiles && begin < end) request(begin);
  find_slot(begin + 1);

  // this lane's row (clamped: rows behind the last repeat it and are not written), turned and cut
  uint4 qh[KS], ql[KS];
  float sc;
  {
    const float4* cs = reinterpret_cast<const float4*>(p.tab + (size_t)(u.n + depth_of(tree, node, p.n)) * (D / 2));
    unsigned top = 0;
#pragma unroll
    for (int x = 0; x < KS; ++x)
      top = max_magnitudes(max_magnitudes(max_magnitudes(raw_q[x].x, raw_q[x].y), max_magnitudes(raw_q[x].z, raw_q[x].w)), top);
    top = max_magnitudes(top, __shfl_xor(top, 32, 64));
    float inverse;
    const float scale = row_scale(top, inverse);
    sc = p.scale_log2e * inverse;
#pragma unroll
    for (int x = 0; x < KS; ++x) turn_cut(raw_q[x], scale, cs[(x * 2 + hi) * 2], cs[(x * 2 + hi) * 2 + 1], qh[x], ql[x]);
  }

  f32x16_t o[DB];
  float ref = REF_NONE, sum = 0.f;
#pragma unroll
  for (int d = 0; d < DB; ++d) o[d] = f32x16_t{};
  auto col_of = [&](int i) { return (i >> 2) * 8 + hi * 4 + (i & 3); };      // column, inside the wave's 32, of element i

  for (int t = begin; t < end; ++t) {
    lds_barrier();                                   // the tile before is done with
    put();                                           // (all of its loads have arrived, and the copies of V before them)
    const bool cached = t < cache_tiles;
    if (t + 1 < end) request(t + 1);
    find_slot(t + 2);
    lds_barrier();
    uint16_t* vt = vs + ((t - begin) & 1) * TILE;
    bool odd = false;
    if (!cached) {
      odd = clear_odd<D>(vt);
    } else if ((t + 1) * TILE_COLS > u.n) {
      clear_cached<D>(vt, t * TILE_COLS, u.n, -1);
      lds_barrier();
    }
    const int col0 = (cached ? t : t - cache_tiles) * TILE_COLS + cg * 32;
    if (col0 >= (cached ? u.n : p.n)) continue;      // (wave-uniform; every wave meets the barriers)
    f32x16_t s = {};
    const int l = anew(lane), k_row = l & 31;
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const int at = (cg * 32 + k_row) * D + ((x * 2 + (l >> 5)) ^ kswz(k_row)) * 8;
      const uint4 h = *reinterpret_cast<const uint4*>(kh + at), low = *reinterpret_cast<const uint4*>(kl + at);
      s = mfma_half(low, qh[x], s);
      s = mfma_half(h, ql[x], s);
      s = mfma_half(h, qh[x], s);
    }
#pragma unroll
    for (int i = 0; i < 16; i += 4) {                // scaled logits
      const float4 f = *reinterpret_cast<const float4*>(col_scale + cg * 32 + col_of(i));
      s[i] *= sc * f.x; s[i + 1] *= sc * f.y; s[i + 2] *= sc * f.z; s[i + 3] *= sc * f.w;
    }
    if (cached) {
      if (col0 + 32 > u.n) {
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = col0 + col_of(i) < u.n ? s[i] : -INFINITY;
      }
    } else {
      const unsigned bits = tree.anc[node][col0 >> 5] >> (hi * 4);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = (bits >> ((i >> 2) * 8 + (i & 3)) & 1) ? s[i] : -INFINITY;
    }
    {
      float top = s[0];
#pragma unroll
      for (int i = 1; i < 16; ++i) top = fmaxf(top, s[i]);
      if (__any(top - ref > 8.0f)) {
        float raised = fmaxf(ref, top);
        raised = fmaxf(raised, __shfl_xor(raised, 32, 64));
        const float by = fast_exp2(ref - raised);
        sum *= by;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] *= by;
        ref = raised;
      }
    }
    if (odd) add_odd_values<DB>(o, Vn + col0 * node_bytes + hi * 8, node_bytes, min(32, p.n - col0), tree.anc[node][col0 >> 5]);
    float add = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i] = fast_exp2(s[i] - ref);
      add += s[i];
    }
    sum += add;
    const int l2 = anew(lane), v_row = (l2 >> 5) * 4 + ((l2 & 15) >> 2), v_piece = ((l2 >> 4) & 1) * 2 + ((l2 >> 1) & 1);
    add_wide_values<D>(o, s, vt + (cg * 32 + v_row) * D + (l2 & 1) * 4, v_piece, vswz(v_row));
  }
  __syncthreads();

  float* so = tr_smem;                               // [CG][ROWS][D + 4]
  float2* sm = reinterpret_cast<float2*>(tr_smem + CG * ROWS * OR);
  leave_wide_sums<D>(o, ref, sum, so, sm, cg * ROWS + rg * 32 + lr, hi);
  __syncthreads();
  finish_rows<D, CG, ROWS>(p, tree, so, sm, unit, tile, slice);
}

// The slices' partial results of one query row, added: a row takes D / 4 lanes.
template <int D>
__global__ __launch_bounds__(256) void tree_merge_kernel(Args p, int rows_per_tile) {
  const int rows = p.n << p.g_bits, unit = blockIdx.y, slices = p.slices;
  const int row = blockIdx.x * (256 / (D / 4)) + threadIdx.x / (D / 4), c = threadIdx.x % (D / 4) * 4;
  if (row >= rows) return;
  const int tile = row / rows_per_tile, r = row % rows_per_tile;
  const float* part = p.scratch + ((size_t)unit * p.row_tiles + tile) * slices * rows_per_tile * (D + 4) + (size_t)r * (D + 4);
  const size_t step = (size_t)rows_per_tile * (D + 4);
  // eight slices at a time, those past the last one empty: a batch's reads are one wait
  constexpr int BATCH = 8;
  float M = REF_NONE, L = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  bool present = true;
  for (int s0 = 0; s0 < slices; s0 += BATCH) {
    float2 ml[BATCH];
    float4 y[BATCH];
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      const float* src = part + min(s0 + x, slices - 1) * step;
      ml[x] = *reinterpret_cast<const float2*>(src + D);
      y[x] = *reinterpret_cast<const float4*>(src + c);
    }
    float top = M;
#pragma unroll
    for (int x = 0; x < BATCH; ++x) top = fmaxf(top, ml[x].x);
    const float by = fast_exp2(M - top);
    L *= by;
    a.x *= by; a.y *= by; a.z *= by; a.w *= by;
    M = top;
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      if (s0 + x < slices) {
        const float f = fast_exp2(ml[x].x - M);
        present = present && !(ml[x].y < 0.f);
        L = fmaf(ml[x].y, f, L);
        a.x = fmaf(y[x].x, f, a.x); a.y = fmaf(y[x].y, f, a.y); a.z = fmaf(y[x].z, f, a.z); a.w = fmaf(y[x].w, f, a.w);
      }
    }
  }
  const int b = unit / p.Hkv, kvh = unit % p.Hkv;
  const size_t at = ((size_t)b * p.n + (row >> p.g_bits)) * p.H + (kvh << p.g_bits) + (row & ((1 << p.g_bits) - 1));
  const float inv = 1.0f / L;
  *reinterpret_cast<float4*>(p.out + at * D + c) =
      present ? make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv) : make_float4(0.f, 0.f, 0.f, 0.f);
  if (c == 0 && p.lse) p.lse[at] = present ? (M + log2f(L)) * LN2 : -INFINITY;
}

// ---------------------------------------------------------------------------------------------
// commit: column sums of the path's rows
// ---------------------------------------------------------------------------------------------
constexpr int CS_ROWS = 64;                          // query rows taken at a time

// Tokens of sequence b's path, -1 if it is none; every thread gets the answer.
__device__ inline int path_length(const Tree& t, int b) {
  const int len = t.path_len[b];
  bool ok = len >= 0 && len <= t.max_len;
  const int i = threadIdx.x;
  if (ok && i < len) {
    const int node = t.path[(size_t)b * t.max_len + i], before = i > 0 ? t.path[(size_t)b * t.max_len + i - 1] : -1;
    ok = node > before && node >= 0 && node < t.n;   // (a parent comes before its child)
    if (ok) ok = t.parents[(size_t)b * t.n + node] == before;
  }
  return __syncthreads_and(ok) ? len : -1;
}

// grid (slices, U).  A column belongs to one lane group of one wave for the whole call, so its accumulator is added to
// without atomics.
template <typename T, int D, bool ROPE>
__global__ __launch_bounds__(TR_THREADS, ROPE ? 2 : 4) void tree_colsum_kernel(Params p, Tree t, int slices, int32_t* __restrict__ status) {
  using O = Ops<T, D>;
  constexpr int QR = q_row_elems<T, D>(), Q_PART = CS_ROWS * QR, BK = O::COLS / 16, ROWB = D * (int)sizeof(T);
  static_assert(TR_THREADS >= MAX_NODES, "one thread per token of the path");
  extern __shared__ __attribute__((aligned(16))) float tr_smem[];
  __shared__ float row_lse[CS_ROWS];
  const int slice = blockIdx.x, unit = blockIdx.y, tid = threadIdx.x, lane = tid & 63, lr = lane & 15, q4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kvh = unit % p.Hkv, b = unit / p.Hkv;
  const Unit u = load_unit<ROPE>(p.meta, p.E, p.R, p.m, p.n_recent, unit);
  const char* Ku = (const char*)p.K + (size_t)unit * p.cap * ROWB;
  const char* Kn = (const char*)t.k + ((size_t)b * t.n * p.Hkv + kvh) * ROWB;
  const size_t node_bytes = (size_t)p.Hkv * ROWB;
  const int found = path_length(t, b), L = max(found, 0);
  const int* path = t.path + (size_t)b * t.max_len;
  if (slice == 0 && tid == 0) {
    p.meta[(size_t)unit * META_STRIDE + META_PATH] = L;
    if (status && kvh == 0) status[b] = found < 0 ? TREEKV_EINVAL : TREEKV_OK;
  }
  if (L == 0) return;
  const int rows = L * p.G;
  // A probability is at most 1, but past 2^20 its logit and the lse, rounded twice, tell nothing of it: it is held to 1 there.
  // Elsewhere it is held to what keeps a sum finite, whatever lse holds (one of another state may be too small).  A NaN
  // adds nothing: what a score has gained it keeps.
  constexpr float ROOM = 0x1p64f;
  const int cache_blocks = (u.columns + O::COLS - 1) / O::COLS, blocks = cache_blocks + (L + O::COLS - 1) / O::COLS;
  const int begin = (int)((long long)blocks * slice / slices), end = (int)((long long)blocks * (slice + 1) / slices);
  const int cap_cols = colsum_part(p.cap);
  unsigned long long* acc = p.pf_colacc + (size_t)unit * colsum_stride(p);
  T* sq = reinterpret_cast<T*>(tr_smem);
  auto load_keys = [&](typename O::Keys& k, int blk) __attribute__((always_inline)) {
    if (blk < cache_blocks && !ROPE) {
      const char* base = Ku + (size_t)blk * (O::COLS * ROWB);
      const int last = p.cap - 1 - blk * O::COLS;
#pragma unroll
      for (int bk = 0; bk < BK; ++bk) O::load_k(k, bk, base, (unsigned)min(bk * 16 + lr, last) * ROWB + q4 * 16);
    } else {
#pragma unroll
      for (int bk = 0; bk < BK; ++bk) {
        const int c = (blk < cache_blocks ? blk : blk - cache_blocks) * O::COLS + bk * 16 + lr;
        const char* row = blk < cache_blocks ? Ku + (size_t)slot_at(u, p.budget, p.n_sink, p.m, p.n_recent, min(c, u.n - 1)) * ROWB
                                             : Kn + path[min(c, L - 1)] * node_bytes;
        O::load_k(k, bk, row, q4 * 16);
      }
    }
  };
  for (int r0 = 0; r0 < rows; r0 += CS_ROWS) {
    const int here = min(CS_ROWS, rows - r0), tiles = (here + 15) / 16;
    __syncthreads();                                 // the rows before are done with
    auto row_of = [&](int r, const T*& src, int& i) {
      r = min(r0 + r, rows - 1);
      i = r / p.G;
      src = (const T*)t.q + (((size_t)b * t.n + path[i]) * p.H + kvh * p.G + r % p.G) * D;
    };
    if constexpr (ROPE) {
      stage_turned<T, D>(sq, tiles * 16, Q_PART, p.rope_tab, [&](int r, const T*& src, int& pos) {
        row_of(r, src, pos);
        pos += u.n;
      });
    } else {
      constexpr int PIECES = D / Storage<T>::EPL;
      for (int x = tid; x < tiles * 16 * PIECES; x += TR_THREADS) {
        const T* src;
        int i;
        row_of(x / PIECES, src, i);
        *reinterpret_cast<uint4*>(sq + (x / PIECES) * QR + (x % PIECES) * Storage<T>::EPL) = reinterpret_cast<const uint4*>(src)[x % PIECES];
      }
    }
    if (tid < CS_ROWS) {
      const int r = min(r0 + tid, rows - 1), i = r / p.G;
      row_lse[tid] = t.lse[((size_t)b * t.n + path[i]) * p.H + kvh * p.G + r % p.G] * LOG2E;
    }
    __syncthreads();
    typename O::Keys k, next_k;
    if (begin + wave < end) load_keys(k, begin + wave);
    for (int blk = begin + wave; blk < end; blk += TR_WAVES) {
      const bool cached = blk < cache_blocks;
      const int col0 = (cached ? blk : blk - cache_blocks) * O::COLS;
      if (blk + TR_WAVES < end) load_keys(next_k, blk + TR_WAVES);
      int pos[BK];
#pragma unroll
      for (int bk = 0; bk < BK; ++bk) {
        const int c = col0 + bk * 16 + lr;
        pos[bk] = cached ? min(c, u.n - 1) : u.n + min(c, L - 1);
      }
      float col_sum[O::NCOL];
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) col_sum[j] = 0.f;
      for (int tile = 0; tile < tiles; ++tile) {
        typename O::Logits s[1];
        if constexpr (ROPE) {
          turned_logits<D, 1>(s, k, p.rope_tab, pos, sq + (tile * 16 + lr) * QR, Q_PART, q4);
        } else {
          typename O::Query q;
          O::load_q(q, sq + (tile * 16 + lr) * QR, q4);
          logits<D>(s[0], k, q);
        }
        const int r = r0 + tile * 16 + lr, i = r / p.G;
        const float l2 = row_lse[tile * 16 + lr];
        const float most = fabsf(l2) > 0x1p20f ? 1.0f : ROOM;
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j) {
          const int c = col0 + O::col(q4, j);
          const bool seen = r < rows && (cached ? c < u.columns && c != u.hole : c <= i);
          const float e = fast_exp2(fmaf(O::at(s[0], j), p.scale_log2e, -l2));
          col_sum[j] += seen ? fminf(fmaxf(e, 0.f), most) : 0.f;       // (the larger of a NaN and 0 is 0)
        }
      }
      float mine = 0.f;                              // lane lr of a group passes on the group's column lr
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) {
        const float x = group_sum<16>(col_sum[j]);
        mine = lr == j ? x : mine;
      }
      const int c = col0 + O::col(q4, lr & (O::NCOL - 1));
      if (lr < O::NCOL && (cached ? c < u.columns && c != u.hole : c < L)) {
        const int slot = ROPE && cached ? slot_at(u, p.budget, p.n_sink, p.m, p.n_recent, c) : c;
        unsigned long long* a = acc + (cached ? slot : cap_cols + c);
        // fp32 sums in the accumulators' low words (fixed point, which the chunk path's atomics ask for, would cut those below
        // 2^-16 short); zero between calls
        *a = __float_as_uint(r0 == 0 ? mine : __uint_as_float((unsigned)*a) + mine);
      }
      k = next_k;
    }
  }
}

int block_cols(const Params& p) { return p.dtype == TREEKV_BF16 ? 32 : 16; }

// Rows of a workgroup, and slices so that there is a workgroup for each of the 256 compute units but no second round.  16 rows
// run fastest where that leaves three slices or more (or there are few rows), 32 where it fills no more than one round, else
// 128 that share the tiles' way from memory.  us a call, bf16 x 128 unless noted, rows/slices:
//   units x rows, slots   8 x 104, 2048  16/4 14.5, 32/8 16.1, 128/16 20.9;   8 x 32  16/9 12.5, 32/9 15.0;   2 x 512, 4096  16/4 19.0, 32/8 19.1
//   16 x 104, 2048  16/2 19.1, 32/4 18.6;   32 x 104  16/1 24.0, 32/2 23.2, 128/8 26.6;   64 x 52  16/1 24.4, 32/2 23.5
//   128 x 24, 1024  16/1 16.1, 32/1 18.9;   256 x 32, 2048  16/1 62.6, 32/1 54.4;   128 x 64  16/1 51.9, 32/1 32.7, 128/1 63
//   128 x 128, 4096  32/1 107, 128/2 90;   8 x 2048, 2048  32/1 68, 128/2 59, 128/1 79;   128 x 256, 4096  32/1 200, 128/1 146
//   x 64: 128 x 128, 4096  32/1 62.1, 128/2 61.9;   8 x 2048, 2048  32/1 48.6, 128/2 47.9;   256 x 48, 2048  32/1 39.4
// Positions re-assigned, bf16: 16 likewise, else the 64 rows for which the keys are turned once (two workgroups a compute unit):
//   64 x 4, 2048  16/4 27.6, 64/8 39.1;   256 x 16  16/1 77, 64/2 103;   64 x 30  16/2 38.0, 64/8 41.1;   128 x 30  16/1 59.7, 64/4 60.1
//   8 x 104  16/4 24.4, 64/17 30.2;   16 x 52  16/4 24.7, 64/17 31.7;   32 x 52  16/2 36.6, 64/16 35.2;   64 x 52  16/1 57.7, 64/8 45.0
//   x 64: 64 x 4  16/4 18.1, 64/8 24.9;   8 x 104  16/4 16.3, 64/32 22.2;   32 x 52  16/2 23.4, 64/16 22.8;   64 x 52  16/1 32.8, 64/8 27.5
//   128 x 30  16/1 33.1, 64/4 37.1;   256 x 16  16/1 37.9, 64/2 59.6;   256 x 48  16/1 102, 64/2 64.4;   32 x 160, 1024  16/1 35.7, 64/5 23.8
// fp32 storage has 16 and 32 rows and the same rule, which takes the better of the two or one within 7 % of it, but for 16 x 256 and
// 256 x 48 rows, where 32 rows are up to 15 % slower.  Positions as they are, then re-assigned in brackets:
//   8 x 16, 2048  16/17 14.6, 32/17 17.4 (16.4, 20.0);   8 x 104  16/4 22.9, 32/8 24.0 (28.3, 27.4)
//   64 x 16  16/4 28.6, 32/4 37.6 (35.2, 43.1);   64 x 52  16/1 57.1, 32/2 61.1 (76.9, 65.8);   256 x 16  16/1 95, 32/1 107 (109, 136)
//   128 x 60, 1024  16/1 63.9, 32/1 58.8 (85.9, 62.9);   16 x 256  16/1 33.6, 32/2 38.5 (42.5, 39.6);   256 x 48  16/1 100, 32/1 111 (135, 128)
//   x 64: 64 x 16, 2048  16/4 18.4, 32/4 20.9 (22.4, 26.7);   64 x 52  16/1 31.5, 32/2 29.0 (40.6, 38.0)
//   128 x 60, 1024  16/1 29.6, 32/1 26.5 (39.7, 34.9);   16 x 256  16/1 18.2, 32/2 20.4 (24.3, 23.9);   256 x 48  16/1 51.7, 32/1 52.7 (65.1, 72.7)
Shape attend_shape(const Params& p, int n) {
  const int rows = n * p.G, tiles16 = (rows + 15) / 16, tiles32 = (rows + 31) / 32, chip = 256, cols = block_cols(p);
  Shape s;
  const bool bf16 = p.dtype == TREEKV_BF16, turned = bf16 && (p.flags & TREEKV_POSITION_RERANK) != 0;
  if (rows <= 16 || (long long)p.U * tiles16 <= (rows <= 32 ? chip : chip / 3)) s.rows_per_tile = 16;
  else if (turned) s.rows_per_tile = TURN_ROWS;
  else s.rows_per_tile = !bf16 || rows <= 64 || (long long)p.U * tiles32 <= chip ? 32 : 128;
  s.row_tiles = (rows + s.rows_per_tile - 1) / s.rows_per_tile;
  // a wave has a block of columns at least, the large workgroup a tile
  const int blocks = (p.cap + cols - 1) / cols + (n + cols - 1) / cols, tiles = (p.cap + TILE_COLS - 1) / TILE_COLS + (n + TILE_COLS - 1) / TILE_COLS;
  const bool staged = s.rows_per_tile >= TURN_ROWS;
  const int most = staged ? tiles : (blocks + TR_WAVES - 1) / TR_WAVES;
  const long long fit = (s.rows_per_tile == TURN_ROWS ? 2 * chip : chip) / ((long long)p.U * s.row_tiles);
  s.slices = fit < 1 ? 1 : fit < most ? (int)fit : most;
  return s;
}

template <int D>
int launch_merge(const Shape& s, const Args& a, hipStream_t st) {
  if (s.slices > 1) {
    constexpr int PER = 256 / (D / 4);
    hipLaunchKernelGGL(tree_merge_kernel<D>, dim3(((a.n << a.g_bits) + PER - 1) / PER, a.U), dim3(256), 0, st, a, s.rows_per_tile);
  }
  return finish_launch();
}
template <typename T, int D, int RB, bool ROPE>
int launch_attend_rb(const Shape& s, const Args& a, hipStream_t st) {
  const size_t sums = (size_t)TR_WAVES * RB * 16 * ((D + 4) * sizeof(float) + sizeof(float2));
  const size_t queries = ROPE ? (size_t)Ops<T, D>::QPARTS * RB * 16 * q_row_elems<T, D>() * sizeof(T) : 0;
  const size_t lds = sums > queries ? sums : queries;
  auto kernel = tree_attend_kernel<T, D, RB, ROPE>;
  if (hip_failed(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds))) return TREEKV_EHIP;
  const int items = s.row_tiles * s.slices * a.U;
  hipLaunchKernelGGL(kernel, dim3((items + 7) / 8 * 8), dim3(TR_THREADS), lds, st, a);
  return launch_merge<D>(s, a, st);
}
template <int D>
int launch_attend_tiled(const Shape& s, const Args& a, hipStream_t st) {
  const size_t sums = (size_t)TR_WAVES * 32 * ((D + 4) * sizeof(float) + sizeof(float2)), stages = (size_t)2 * STAGES * TILE_COLS * D * 2;
  const size_t lds = sums > stages ? sums : stages;
  auto kernel = tree_attend_tiled_kernel<D>;
  if (hip_failed(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds))) return TREEKV_EHIP;
  const int items = s.row_tiles * s.slices * a.U;
  hipLaunchKernelGGL(kernel, dim3((items + 7) / 8 * 8), dim3(TR_THREADS), lds, st, a);
  return launch_merge<D>(s, a, st);
}
template <int D>
int launch_attend_turned(const Shape& s, const Args& a, hipStream_t st) {
  const size_t sums = (size_t)2 * TURN_ROWS * ((D + 4) * sizeof(float) + sizeof(float2)), tile = (size_t)4 * TILE_COLS * D * 2;
  const size_t lds = sums > tile ? sums : tile;
  auto kernel = tree_attend_turned_kernel<D>;
  if (hip_failed(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds))) return TREEKV_EHIP;
  const int items = s.row_tiles * s.slices * a.U;
  hipLaunchKernelGGL(kernel, dim3((items + 7) / 8 * 8), dim3(TURN_THREADS), lds, st, a);
  return launch_merge<D>(s, a, st);
}
template <typename T, int D>
int launch_attend_d(const Params& p, const Tree& t, float* out, float* lse, float* scratch, hipStream_t st) {
  const Shape s = attend_shape(p, t.n);
  const bool rope = (p.flags & TREEKV_POSITION_RERANK) != 0;
  const Args a = {p.K, p.V, p.meta, p.E, p.R, p.rope_tab, t.q, t.k, t.v, t.parents, out, lse, scratch, p.budget, p.cap, p.n_sink,
                  p.n_recent, p.m, p.U, p.H, p.Hkv, p.G == 1 ? 0 : p.G == 2 ? 1 : p.G == 4 ? 2 : 3, t.n, s.row_tiles, s.slices, p.scale_log2e};
  if constexpr (sizeof(T) == 2) {
    if (s.rows_per_tile == 128) return launch_attend_tiled<D>(s, a, st);
    if (s.rows_per_tile == TURN_ROWS) return launch_attend_turned<D>(s, a, st);
  }
  if (s.rows_per_tile == 16) return rope ? launch_attend_rb<T, D, 1, true>(s, a, st) : launch_attend_rb<T, D, 1, false>(s, a, st);
  if constexpr (sizeof(T) == 4) {
    if (rope) return launch_attend_rb<T, D, 2, true>(s, a, st);
  }
  return launch_attend_rb<T, D, 2, false>(s, a, st);
}

template <typename T, int D, bool ROPE>
int launch_colsums_d(const Params& p, const Tree& t, int32_t* status, hipStream_t st) {
  const size_t lds = (size_t)(ROPE ? Ops<T, D>::QPARTS : 1) * CS_ROWS * q_row_elems<T, D>() * sizeof(T);
  // as many workgroups as run at once, two on each of the 256 compute units or, where keys are turned in 235 registers, one
  // (64 units x 16 rows into 2048 slots: 22.6 us, 28.6 with two rounds), each wave with a block of columns at least
  const int cols = block_cols(p), blocks = (p.cap + cols - 1) / cols + (t.max_len + cols - 1) / cols;
  const int most = (blocks + TR_WAVES - 1) / TR_WAVES, fit = (ROPE && sizeof(T) == 2 ? 256 : 512) / p.U, slices = fit < 1 ? 1 : fit < most ? fit : most;
  auto kernel = tree_colsum_kernel<T, D, ROPE>;
  if (lds > 48 * 1024 &&
      hip_failed(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)))
    return TREEKV_EHIP;
  hipLaunchKernelGGL(kernel, dim3(slices, p.U), dim3(TR_THREADS), lds, st, p, t, slices, status);
  return finish_launch();
}
template <typename T, int D>
int launch_colsums_t(const Params& p, const Tree& t, int32_t* status, hipStream_t st) {
  return (p.flags & TREEKV_POSITION_RERANK) ? launch_colsums_d<T, D, true>(p, t, status, st) : launch_colsums_d<T, D, false>(p, t, status, st);
}

}  // namespace

size_t tree_scratch_bytes(const Params& p, int n) {
  const Shape s = attend_shape(p, n);
  return s.slices > 1 ? align_up((size_t)p.U * s.row_tiles * s.slices * s.rows_per_tile * (p.D + 4) * sizeof(float)) : 0;
}

int launch_tree_attend(const Params& p, const Tree& t, float* out, float* lse, void* scratch, hipStream_t s) {
  float* sc = static_cast<float*>(scratch);
  if (p.dtype == TREEKV_F32) return p.D == 128 ? launch_attend_d<float, 128>(p, t, out, lse, sc, s) : launch_attend_d<float, 64>(p, t, out, lse, sc, s);
  return p.D == 128 ? launch_attend_d<uint16_t, 128>(p, t, out, lse, sc, s) : launch_attend_d<uint16_t, 64>(p, t, out, lse, sc, s);
}

int launch_tree_colsums(const Params& p, const Tree& t, int32_t* status, hipStream_t s) {
  if (p.dtype == TREEKV_F32) return p.D == 128 ? launch_colsums_t<float, 128>(p, t, status, s) : launch_colsums_t<float, 64>(p, t, status, s);
  return p.D == 128 ? launch_colsums_t<uint16_t, 128>(p, t, status, s) : launch_colsums_t<uint16_t, 64>(p, t, status, s);
}

}  // namespace tkv
