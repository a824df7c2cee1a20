// A paged cache for gfx950: treekv_paged_append and treekv_paged_attend.
//
// attend   o_i = sum over j <= i of p_ij v_j, p_ij = exp(q_i k_j * scale - lse_i), over a sequence's pages.  The G query heads
//          of a KV head and the sequence's n new tokens are the rows of one matrix product, in tiles of 16 or 32; columns are
//          slots.  A softmax in one pass: the reference of a row's exponentials is raised where a logit passes it by 2^8, sums
//          are fp32.  With bf16 storage P enters the second product rounded to bf16 (2^-8 of each probability at most, where the
//          output is rounded by as much again); the sum beside it takes the unrounded ones.  Two parts, as a prefill chunk's outputs
//          in fp32 have them, would be half as many products again, in what is bound by products.  Against 64 bits the output is off
//          by 1.9 to 2.1e-3 of its size in place of the 1.7e-3 of its own rounding.
//          A page holds a multiple of 16 rows, so 16 columns lie in one page: one address for the wave and a lane's offset.
// shares   Few rows leave most of the chip idle, so the columns of the whole batch are cut into equal shares, which the device
//          works out from the lengths: long sequences get more workgroups than short ones.  A sequence's shares are merged by a
//          second kernel.
//          Bound by memory: 16 sequences of 4000 to 16000 tokens, 8 groups of 4 heads, a token each, 117 us, 6.05 TB/s of K and V.
// many     More than 64 rows share K and V through LDS (below).  512 tokens of 8 groups of 4 heads over 32768: 287-305 us, 0.95 PFLOP/s
//          where a large product of the library reaches 1.2.
// weights  the probabilities once more, from kept logits or from q and k, by each row's reference and sum, summed down the rows: a
//          column belongs to one wave, so the sum needs no atomics and repeats bit for bit.

#include "treekv_matrix.h"
#include "treekv_paged.h"
#include "treekv_shares.h"

// Multiply-adds only where they are written: a logit has to be rounded like the reference that it was compared to (fused with the
// subtraction of the reference it would differ by what the reference lost, 2^7 from 2^31 on).
#pragma clang fp contract(off)

namespace tkv {

namespace {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;

__device__ inline unsigned narrow2(float a, float b) {
  const f32x2_t v = {a, b};
  return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2_t));
}

// ---- append ------------------------------------------------------------------------------------
// A workgroup takes TOK tokens: their places first, then the rows in 16-byte pieces, then weights and positions, whose TOK
// words of a head are neighbours.
template <int TOK>
__global__ __launch_bounds__(PA_THREADS) void append_kernel(Pages p, const char* k, const char* v, int64_t k_far, int64_t v_far,
                                                            const int32_t* starts, int tokens, const int32_t* positions,
                                                            int32_t* status, int piece_bits) {
  __shared__ int at_b[TOK], at_slot[TOK], at_page[TOK], odd;       // odd: starts do not ascend; halving them does not find a row's sequence
  const int tid = threadIdx.x, t0 = (int)blockIdx.x * TOK;
  if (tid < TOK) {
    const int t = t0 + tid;
    int b = -1, slot = 0, page = -1;
    if (t < tokens) {
      int lo = 0, hi = p.B - 1;                        // the first sequence that ends behind t
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid + 1] > t) hi = mid; else lo = mid + 1;
      }
      const Seq s = load_seq(p, starts, tokens, tokens, lo);
      if (t >= s.first && t < s.first + s.n) {
        b = lo;
        slot = s.len - s.n + (t - s.first);
        page = p.table[(size_t)b * p.width + (slot >> p.bits)];
        if (page < 0 || page >= p.pages) page = -1;
      }
    }
    at_b[tid] = b; at_slot[tid] = slot; at_page[tid] = page;
  } else if (tid >> 6 == 1) {
    bool ascend = true;
    for (int b = tid & 63; b < p.B; b += 64) ascend &= ascends(starts[b], starts[b + 1], tokens);
    ascend = __all(ascend);
    if (tid == 64) odd = !ascend;
  }
  __syncthreads();
  if (__builtin_expect(odd, 0)) {
    if (tid < TOK) at_b[tid] = -1;
    __syncthreads();
    if (tid < 64) {
      int end = 0;
      for (int b0 = 0; b0 < p.B; b0 += 64) {
        const int b = b0 + tid;
        const Seq s = load_seqs(p, starts, tokens, tokens, b0, end);
        for (int i = 0; i < TOK; ++i) {
          const int t = t0 + i;
          if (t >= tokens || t < s.first || t >= s.first + s.n) continue;          // (no row has two sequences)
          const int slot = s.len - s.n + (t - s.first), page = p.table[(size_t)b * p.width + (slot >> p.bits)];
          at_b[i] = b; at_slot[i] = slot; at_page[i] = page < p.pages ? page : -1;
        }
      }
    }
    __syncthreads();
  }
  if (blockIdx.x == 0 && status) write_status(p, starts, tokens, tokens, odd, status, PA_THREADS);
  const int row_pieces = p.Hkv << piece_bits, all = 2 * row_pieces * TOK;
  for (int x = tid; x < all; x += PA_THREADS) {
    const int i = x / (2 * row_pieces);
    int y = x - i * 2 * row_pieces;
    const bool second = y >= row_pieces;
    if (second) y -= row_pieces;
    if (at_b[i] < 0 || at_page[i] < 0) continue;
    const char* src = (second ? v + (t0 + i) * v_far : k + (t0 + i) * k_far) + (size_t)y * 16;
    const size_t row = pool_row(p, at_page[i], y >> piece_bits, at_slot[i]);
    char* dst = (second ? p.v : p.k) + (((row << piece_bits) + (y & ((1 << piece_bits) - 1))) << 4);
    *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(src);
  }
  if (p.weights)
    for (int x = tid; x < p.Hkv * TOK; x += PA_THREADS) {
      const int h = x / TOK, i = x % TOK;
      if (at_b[i] < 0) continue;
      const size_t at = track_row(p, at_b[i], h) + at_slot[i];
      p.weights[at] = 0.f;
      p.positions[at] = positions[t0 + i];
    }
}

// ---- attend ------------------------------------------------------------------------------------
struct Attend {
  Pages p;
  const int32_t* starts;
  const char* q;
  int64_t q_far;                             // bytes from one token's heads to the next one's
  char* out;
  float *lse, *part;
  float2* stat;                              // for the weights: a row's reference and 1 / its sum (infinity and 0 if it adds nothing)
  int32_t* status;
  float* gains;                              // splits of a column's rows: [split][sequence][KV head][cap]
  float* logits;                             // few rows and weights: scaled logits, [sequence][KV head][row][cap]
  int tokens, longest, tiles, shares, rows;  // row tiles of the longest sequence; shares the columns are cut into; rows of a tile
  int least_rows, most_rows;                 // sequences with others are not this kernel's
  float scale_log2e;
  bool wide, sparse;                         // more columns than 32 bits count; how partial results are numbered
};

// The columns of all sequences with new tokens lie one after the other (each sequence's rounded up to whole blocks), and are cut
// into shares of `size`.  Few rows over many columns: a workgroup takes one share, whatever sequences it runs through.  Many rows,
// where there are row tiles to go round, and small shares: a sequence's shares start at its first token, so that each is of one
// sequence (its `own`).
struct Run : Runs {
  int b, length;             // a sequence with columns, and their number
  long long start;           // where they start
};
__device__ inline int columns_in(const Attend& a, const Seq& s) {
  const int rows = s.n * a.p.G;
  return rows >= a.least_rows && rows <= a.most_rows ? (s.len + 31) & ~31 : 0;
}
// (Of one that begins before the end of an earlier one's rows too: its columns are counted like the others', and passed over.)
__device__ inline int columns_of_seq(const Attend& a, int b) {
  return b < a.p.B ? columns_in(a, load_seq(a.p, a.starts, a.tokens, a.longest, b)) : 0;
}
__device__ inline long long uniform64(long long x) {
  return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)x));
}
// Sums up to each lane, and the last one's; `wide`: past 32 bits.
__device__ inline long long wave_scan(long long x, bool wide, long long& all) {
  const int lane = threadIdx.x & 63;
  if (wide) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const long long y = __shfl_up(x, d, 64);
      if (lane >= d) x += y;
    }
    all = uniform64(__shfl(x, 63, 64));
    return x;
  }
  int v = (int)x;
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, true);      // within 16 lanes (row_shr)
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, true);
  const int r0 = __builtin_amdgcn_readlane(v, 15), r1 = r0 + __builtin_amdgcn_readlane(v, 31), r2 = r1 + __builtin_amdgcn_readlane(v, 47);
  v += lane < 16 ? 0 : lane < 32 ? r0 : lane < 48 ? r1 : r2;
  all = __builtin_amdgcn_readlane(v, 63);
  return v;
}
// What find_run asks of the lengths: the cut, and this lane's sequence among the first 64.
struct Columns : Cut {
  int length;
  bool odd;                  // starts do not ascend
};
__device__ inline Columns columns_of(const Attend& a, bool tiled) {
  const int lane = threadIdx.x & 63;
  Columns c;
  bool ascend = true;
  c.length = 0;
  if (lane < a.p.B) {
    const Seq s = load_seq(a.p, a.starts, a.tokens, a.longest, lane);
    c.length = columns_in(a, s);
    ascend = s.ascends;
  }
  long long total, mine = c.length;
  for (int b = 64 + lane; b < a.p.B; b += 64) {
    const Seq s = load_seq(a.p, a.starts, a.tokens, a.longest, b);
    mine += columns_in(a, s);
    ascend &= s.ascends;
  }
  c.odd = !__all(ascend);
  wave_scan(mine, a.wide, total);
  static_cast<Cut&>(c) = cut_columns(total, a.shares, a.p.B, tiled, a.wide, [&](int size) {
    long long count;
    wave_scan(shares_in(c.length, size), false, count);
    return (int)count;
  });
  return c;
}
// The sequence that holds column `at` of all (want_b < 0), or sequence want_b.  One share a sequence at least: `own`.
__device__ inline bool find_run(const Attend& a, const Columns& c, long long at, int want_b, Run& run) {
  const int lane = threadIdx.x & 63, size = c.size;
  const bool own = c.own;
  long long before = 0;
  for (int b0 = 0; b0 < a.p.B; b0 += 64) {
    const int length = b0 ? columns_of_seq(a, b0 + lane) : c.length, mine = own ? shares_in(length, size) : length;
    long long all;
    const long long sum = wave_scan(mine, a.wide, all);
    const unsigned long long hit = __ballot(want_b < 0 ? mine > 0 && before + sum > at : b0 + lane == want_b);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;
      run.b = b0 + l;
      run.length = __builtin_amdgcn_readlane(length, l);
      const long long start = sum - mine;
      run.start = before + (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(start >> 32), l) << 32 |
                                       (unsigned)__builtin_amdgcn_readlane((int)start, l));
      static_cast<Runs&>(run) = runs_of(c, a.wide, run.start, run.length);
      return true;
    }
    before += all;
  }
  return false;
}
// Whether its rows are an earlier sequence's.
__device__ inline bool refused(const Attend& a, const Columns& c, int b, const Seq& s) {
  return __builtin_expect(c.odd, 0) && begins_inside(a.starts, a.tokens, b, s.first);
}
// Where a sequence's partial results lie, if it has any.  MERGED: only what is merged has them.
template <bool MERGED>
__device__ inline int first_part(const Attend& a, const Columns& c, const Run& run) {
  long long before = run.start;                        // columns of earlier sequences
  if (MERGED && a.sparse && c.own && run.count > 1) {
    const int lane = threadIdx.x & 63;
    long long mine = 0;
    for (int b = lane; b < run.b; b += 64) mine += columns_of_seq(a, b);
    wave_scan(mine, a.wide, before);
  }
  return part_of_first(c, a.wide, MERGED && a.sparse, run, before, run.b);
}

template <int D>
__device__ inline void add_rounded(f32x4_t (&o)[D / 16], const typename Ops<uint16_t, D>::Values& v,
                                   const typename Ops<uint16_t, D>::Logits& p) {
  const uint4 h = make_uint4(narrow2(p.x[0][0], p.x[0][1]), narrow2(p.x[0][2], p.x[0][3]),
                             narrow2(p.x[1][0], p.x[1][1]), narrow2(p.x[1][2], p.x[1][3]));
#pragma unroll
  for (int e = 0; e < D / 16; ++e) o[e] = mfma_bf16(Ops<uint16_t, D>::dim(v, e), h, o[e]);
}
template <int D>
__device__ inline void add_rounded(f32x4_t (&o)[D / 16], const typename Ops<float, D>::Values& v,
                                   const typename Ops<float, D>::Logits& p) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
#pragma unroll
    for (int e = 0; e < D / 16; ++e) o[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v.x[j][e], p.x[0][j], o[e], 0, 0, 0);
}

// A finished row's four dimensions from c: the sums over the softmax's sum.
__device__ inline void store4(char* out, size_t at, const float4& a, float inv, uint16_t) {
  *reinterpret_cast<uint2*>(out + at * 2) = make_uint2(narrow2(a.x * inv, a.y * inv), narrow2(a.z * inv, a.w * inv));
}
__device__ inline void store4(char* out, size_t at, const float4& a, float inv, float) {
  *reinterpret_cast<float4*>(out + at * 4) = make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
}
__device__ inline float2 stat_of_sums(float M, float L) { return L > 0.f ? make_float2(M, 1.0f / L) : make_float2(INFINITY, 0.f); }
__device__ inline void finish_sums(const Attend& a, size_t at, float M, float L) {
  if (a.lse) a.lse[at] = !(L == 0.f) ? (M + log2f(L)) * LN2 : -INFINITY;
  if (a.stat) a.stat[at] = stat_of_sums(M, L);
}
template <typename T, int D>
__device__ inline void finish_row(const Attend& a, const Seq& s, int h, int row, int c, const float4& o, float M, float L) {
  const size_t at = (size_t)(s.first + row / a.p.G) * a.p.H + h * a.p.G + row % a.p.G;
  const bool any = !(L == 0.f);                          // (a sum that is a NaN stays one)
  store4(a.out, at * D + c, any ? o : make_float4(0.f, 0.f, 0.f, 0.f), any ? 1.0f / L : 0.f, T());
  if (c == 0) finish_sums(a, at, M, L);
}

// grid: shares of the columns x KV heads x row tiles.  RB: blocks of 16 rows.
// WEIGH (one tile only): the logits are kept for the weights.
template <typename T, int D, int RB, bool WEIGH>
__global__ __launch_bounds__(PA_THREADS, 2) void attend_kernel(Attend a) {
  using O = Ops<T, D>;
  constexpr int ROWS = RB * 16, DPL = O::DPL, OR = D + 4, BK = O::COLS / 16, COLS = O::COLS, ROWB = D * (int)sizeof(T);
  extern __shared__ __attribute__((aligned(16))) float pa_smem[];
  const Pages& p = a.p;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, q4 = lane >> 4;
  const int tile = (int)(blockIdx.x % a.tiles), rest = (int)(blockIdx.x / a.tiles), h = rest % p.Hkv, w = rest / p.Hkv;
  const Columns columns = columns_of(a, false);
  if (blockIdx.x == 0 && a.status) write_status(p, a.starts, a.tokens, a.longest, columns.odd, a.status, PA_THREADS);
  const int size = columns.size;
  const bool own = columns.own;
  const long long share_end = own ? w + 1 : (long long)(w + 1) * size;
  Run run;
#pragma unroll 1
  for (long long from = own ? w : (long long)w * size; from < share_end && find_run(a, columns, from, -1, run);
       from = own ? share_end : run.start + run.length) {
    const Seq s = load_seq(p, a.starts, a.tokens, a.longest, run.b);
    const int rows = s.n * p.G, row0 = tile * ROWS;
    if (row0 >= rows || refused(a, columns, run.b, s)) continue;
    const int old = s.len - s.n, part0 = first_part<!WEIGH>(a, columns, run) + part_at(!WEIGH && a.sparse, w - run.first);
    // columns: what the tile's first row sees all rows see, behind what its last row sees there is nothing for it
    const int all_see = old + row0 / p.G + 1, end = old + (min(row0 + ROWS, rows) - 1) / p.G + 1;
    const int lo = own ? (w - run.first) * size : (int)(from - run.start);
    const int hi = (int)min((long long)end, own ? (long long)lo + size : share_end - run.start);

    typename O::Query q[RB];
    int see[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const int row = min(row0 + rb * 16 + r, rows - 1), i = row / p.G;
      see[rb] = old + i + 1;
      O::load_q(q[rb], reinterpret_cast<const T*>(a.q + (s.first + i) * a.q_far) + (size_t)(h * p.G + row - i * p.G) * D, q4);
    }
    f32x4_t o[RB][D / 16];
    float ref[RB], sum[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      ref[rb] = REF_NONE;
      sum[rb] = 0.f;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) o[rb][e] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    const int32_t* table = p.table + (size_t)run.b * p.width;
    const int in_page = (1 << p.bits) - 1;

    // the pages of the wave's next AT_ONCE blocks, 16 columns to a lane (a lookup per block would be waited for before its rows)
    constexpr int AT_ONCE = 64 / BK;
    auto look_up = [&](int c0) {
      const int c = c0 + lane / BK * (PA_WAVES * COLS) + lane % BK * 16;
      const int page = c < hi ? table[c >> p.bits] : -1;
      return page >= 0 && page < p.pages ? page : -1;
    };
    int left = 0, pages = -1;
    // a block's place: the bytes of its quarters' rows, which of them are there
    struct Block {
      size_t at[BK];
      bool there[BK];
    };
    auto next_block = [&](int c0) {
      if (left % AT_ONCE == 0) {
        pages = look_up(c0);
        left = 0;
      }
      Block b;
#pragma unroll
      for (int x = 0; x < BK; ++x) {
        const int page = __builtin_amdgcn_readlane(pages, left * BK + x);
        b.there[x] = page >= 0;
        b.at[x] = ((((size_t)max(page, 0) * p.Hkv + h) << p.bits) + ((c0 + 16 * x) & in_page)) * ROWB;
      }
      ++left;
      return b;
    };
    // keys are asked for a block ahead, values before the block's logits are formed; up to 16 rows are one tile, whose values nobody
    // else reads (past the caches 16 sequences of 16000 tokens take 117 us in place of 130, with weights 154 in place of 164; the keys
    // too: 116 and 160, and 45 in place of 41 where 134 MB lie in the memory-side cache)
    typename O::Keys k;
    Block to_come = next_block(lo + wave * COLS);
#pragma unroll
    for (int x = 0; x < BK; ++x) O::load_k(k, x, p.k + to_come.at[x], r * ROWB + q4 * 16);
#pragma unroll 1
    for (int c0 = lo + wave * COLS; c0 < hi; c0 += PA_WAVES * COLS) {
      const Block now = to_come;
      const auto& at = now.at;
      const auto& there = now.there;
      bool whole = c0 + COLS <= all_see;
#pragma unroll
      for (int x = 0; x < BK; ++x) whole &= there[x];
      typename O::Values v;
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) O::template load_v<RB == 1>(v, j, p.v + at[j * BK / O::NCOL], (O::col(q4, j) & 15) * ROWB + r * DPL * (int)sizeof(T));
      typename O::Logits x_of[RB];
      typename O::Keys k_next;
      to_come = next_block(c0 + PA_WAVES * COLS);
#pragma unroll
      for (int x = 0; x < BK; ++x) O::load_k(k_next, x, p.k + to_come.at[x], r * ROWB + q4 * 16);
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) logits<D>(x_of[rb], k, q[rb]);
      k = k_next;
      bool odd = false;
      if (!whole) {
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j)
          if (!there[j * BK / O::NCOL] || c0 + O::col(q4, j) >= hi) O::clear_v(v, j);
        odd = !all_finite<D>(v);
        if (odd) drop_not_finite<D>(v);
      }
#pragma unroll
      for (int rb = 0; rb < RB; ++rb) {
        typename O::Logits& x = x_of[rb];
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j) {
          float& y = O::at(x, j);
          y *= a.scale_log2e;
          if (!whole && (!there[j * BK / O::NCOL] || c0 + O::col(q4, j) >= min(see[rb], hi))) y = -INFINITY;
          mx = fmaxf(mx, y);
        }
        if constexpr (WEIGH) {
          if (rb * 16 + r < rows) {
            float* keep = a.logits + (((size_t)run.b * p.Hkv + h) * a.rows + rb * 16 + r) * p.cap + c0 + 4 * q4;
#pragma unroll
            for (int z = 0; z < BK; ++z)
              if (c0 + 16 * z < hi) *reinterpret_cast<f32x4_t*>(keep + 16 * z) = x.x[z];
          }
        }
        if (__any(mx > ref[rb] + 8.f)) {
          mx = row_max(mx);
          const float to = mx > ref[rb] + 8.f ? mx : ref[rb], f = fast_exp2(ref[rb] - to);
          sum[rb] *= f;
#pragma unroll
          for (int e = 0; e < D / 16; ++e) o[rb][e] *= f;
          ref[rb] = to;
        }
#pragma unroll
        for (int j = 0; j < O::NCOL; ++j) {
          float& y = O::at(x, j);
          y = fast_exp2(y - ref[rb]);
          sum[rb] += y;
        }
        add_rounded<D>(o[rb], v, x);
      }
      if (odd) {
#pragma unroll
        for (int x = 0; x < BK; ++x) {
          if (!there[x]) continue;
          unsigned bits[RB];
#pragma unroll
          for (int rb = 0; rb < RB; ++rb) bits[rb] = (1u << max(0, min(min(see[rb], hi) - c0 - 16 * x, 16))) - 1;
          add_not_finite<T, D, RB>(o, p.v + at[x] + DPL * 4 * q4 * (int)sizeof(T), ROWB, max(0, min(16, hi - c0 - 16 * x)), bits);
        }
      }
    }

    // the waves' sums, [wave][row][D], and references
    float* so = pa_smem;
    float2* sm = reinterpret_cast<float2*>(pa_smem + PA_WAVES * ROWS * OR);
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
      const float total = row_sum(sum[rb]);
      float* row = so + ((size_t)wave * ROWS + rb * 16 + r) * OR;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < D / 16; e += 4)
          *reinterpret_cast<float4*>(row + (4 * q4 + i) * DPL + e) = make_float4(o[rb][e][i], o[rb][e + 1][i], o[rb][e + 2][i], o[rb][e + 3][i]);
      if (q4 == 0) sm[wave * ROWS + rb * 16 + r] = make_float2(ref[rb], total);
    }
    __syncthreads();
    for (int x = tid; x < ROWS * (D / 4); x += PA_THREADS) {
      const int y = x / (D / 4), c = x % (D / 4) * 4;
      if (row0 + y >= rows) break;
      float M = REF_NONE, L = 0.f;
#pragma unroll
      for (int z = 0; z < PA_WAVES; ++z) M = fmaxf(M, sm[z * ROWS + y].x);
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int z = 0; z < PA_WAVES; ++z) {
        const float2 ml = sm[z * ROWS + y];
        const float g = fast_exp2(ml.x - M);
        const float4 u = *reinterpret_cast<const float4*>(so + ((size_t)z * ROWS + y) * OR + c);
        L = fmaf(ml.y, g, L);
        f.x = fmaf(u.x, g, f.x); f.y = fmaf(u.y, g, f.y); f.z = fmaf(u.z, g, f.z); f.w = fmaf(u.w, g, f.w);
      }
      float* part = a.part + (((size_t)part0 * p.Hkv + h) * a.tiles + tile) * ROWS * OR + (size_t)y * OR;
      if (c == 0 && (WEIGH || run.count > 1)) *reinterpret_cast<float2*>(part + D) = make_float2(M, L);
      if (run.count > 1) *reinterpret_cast<float4*>(part + c) = f;
      else finish_row<T, D>(a, s, h, row0 + y, c, f, M, L);
    }
    __syncthreads();                                     // (the sums in LDS make way for the next sequence's)
  }
}

// Shares of a sequence added, four dimensions of a row a thread, `slices` (a power of two up to MERGE_ROWS) groups of threads
// to a row: of MERGE_ROWS / slices rows at once, from row0 on, every `step` rows.
template <int D> constexpr int MERGE_ROWS = PA_THREADS * 4 / D;
struct Merged {
  float4 f[PA_THREADS];
  float2 ml[PA_THREADS];
};
template <typename T, int D, bool MERGED>
__device__ inline void merge_rows(const Attend& a, const Seq& s, const Run& run, int part0, int h, int row0, int step, int slices, Merged& sm) {
  constexpr int OR = D + 4, WIDTH = D / 4;
  const Pages& p = a.p;
  const int rows = s.n * p.G, tid = threadIdx.x, c = tid % WIDTH * 4, slice = tid / WIDTH & (slices - 1);
  for (; row0 < rows; row0 += step) {
    const int row = row0 + tid / WIDTH / slices;
    const size_t far = (size_t)p.Hkv * a.tiles * a.rows * OR;
    const float* part = a.part + (((size_t)part0 * p.Hkv + h) * a.tiles * a.rows + min(row, rows - 1)) * OR;
    constexpr int AT_ONCE = 8;                         // shares on their way together
    float M = REF_NONE, L = 0.f;
    float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z0 = slice; z0 < run.count; z0 += AT_ONCE * slices) {
      float2 ml[AT_ONCE];
      float4 u[AT_ONCE];
#pragma unroll
      for (int z = 0; z < AT_ONCE; ++z) {
        const float* at = part + part_at(MERGED && a.sparse, min(z0 + z * slices, run.count - 1)) * far;
        ml[z] = *reinterpret_cast<const float2*>(at + D);
        u[z] = *reinterpret_cast<const float4*>(at + c);
      }
      float to = M;
#pragma unroll
      for (int z = 0; z < AT_ONCE; ++z) to = fmaxf(to, ml[z].x);
      const float was = fast_exp2(M - to);
      L *= was; f.x *= was; f.y *= was; f.z *= was; f.w *= was;
      M = to;
#pragma unroll
      for (int z = 0; z < AT_ONCE; ++z) {
        if (z0 + z * slices >= run.count) break;
        const float g = fast_exp2(ml[z].x - M);
        L = fmaf(ml[z].y, g, L);
        f.x = fmaf(u[z].x, g, f.x); f.y = fmaf(u[z].y, g, f.y); f.z = fmaf(u[z].z, g, f.z); f.w = fmaf(u[z].w, g, f.w);
      }
    }
    if (slices > 1) {
      __syncthreads();                                 // (the rows before have been read)
      sm.f[tid] = f;
      sm.ml[tid] = make_float2(M, L);
      __syncthreads();
      if (slice == 0) {
        float to = M;
        for (int z = 1; z < slices; ++z) to = fmaxf(to, sm.ml[tid + z * WIDTH].x);
        const float was = fast_exp2(M - to);
        L *= was; f.x *= was; f.y *= was; f.z *= was; f.w *= was;
        M = to;
        for (int z = 1; z < slices; ++z) {
          const float2 ml = sm.ml[tid + z * WIDTH];
          const float4 u = sm.f[tid + z * WIDTH];
          const float g = fast_exp2(ml.x - M);
          L = fmaf(ml.y, g, L);
          f.x = fmaf(u.x, g, f.x); f.y = fmaf(u.y, g, f.y); f.z = fmaf(u.z, g, f.z); f.w = fmaf(u.w, g, f.w);
        }
      }
    }
    if (slice == 0 && row < rows) finish_row<T, D>(a, s, h, row, c, f, M, L);
  }
}
// The tiles of a group (a KV head of a share or of a sequence) run on one XCD, whose L2 then has what they share, and with fewer
// than 8 KV heads on as many XCDs as leaves none idle, as far as there are tiles for them, which another group begins at another
// of them; not where there are four groups or more for each XCD (of `turns` shares or sequences).  (2 KV heads, groups of 8, 2154
// tokens behind 15291: 714 -> 438 us against one XCD for each; the weights of 3084 tokens behind 5208, 2 heads: 105 -> 71 with the
// attention, and their rows shared between workgroups.)
struct Place {
  int group, tile;                             // (maybe behind the last)
};
__host__ __device__ inline int xcds_of_group(int heads, int turns, int tiles) {
  int of = 1;
  while (of < 8 && heads % (8 / of) != 0 && (long long)heads * turns < 4 * (8 / of) && 2 * of <= tiles) of *= 2;
  return of;
}
__device__ inline Place place_of(int heads, int turns, int tiles) {
  const int of = xcds_of_group(heads, turns, tiles), together = 8 / of, each = (tiles + of - 1) / of;       // groups beside each other
  const int x = (int)(blockIdx.x & 7), i = (int)(blockIdx.x >> 3);
  return {i / each * together + x % together, i % each * of + (x / together + i / each) % of};
}
unsigned places(unsigned groups, int heads, int turns, int tiles) {
  const unsigned of = xcds_of_group(heads, turns, tiles), together = 8 / of;
  return (groups + together - 1) / together * ((tiles + of - 1) / of) * 8;
}

// grid: groups of MERGE_ROWS / slices rows x KV heads x sequences.  PACKED: groups of all sequences one after the other x KV heads
// (where the longest sequence's are many more than the others': one of 512 tokens among 31 of one, 56 -> 13 us).
template <typename T, int D, bool PACKED>
__global__ __launch_bounds__(PA_THREADS) void merge_kernel(Attend a, int merge_tiles, int slices, bool tiled) {
  __shared__ Merged sm;
  const Pages& p = a.p;
  const int at_once = MERGE_ROWS<D> / slices, rest = (int)(blockIdx.x / merge_tiles), h = rest % p.Hkv;
  int tile = (int)(blockIdx.x % merge_tiles), b = rest / p.Hkv;
  Columns columns;
  if (PACKED) {
    columns = columns_of(a, tiled);
    const int lane = threadIdx.x & 63;
    unsigned long long hit = 0;
    int end = 0;
    for (int b0 = 0; b0 < p.B && !hit; b0 += 64) {
      Seq s = {0, 0, 0, false, true};
      if (__builtin_expect(columns.odd, 0)) s = load_seqs(p, a.starts, a.tokens, a.longest, b0, end);      // (or there were more groups than the grid has)
      else if (b0 + lane < p.B) s = load_seq(p, a.starts, a.tokens, a.longest, b0 + lane);
      const int mine = columns_in(a, s) ? (s.n * p.G + at_once - 1) / at_once : 0;
      long long all;
      const int sum = (int)wave_scan(mine, false, all);
      hit = __ballot(sum > tile);
      if (hit) {
        b = __ffsll((long long)hit) - 1;
        tile -= __builtin_amdgcn_readlane(sum - mine, b);
        b += b0;
      } else tile -= (int)all;
    }
    if (!hit) return;
  }
  const Seq s = load_seq(p, a.starts, a.tokens, a.longest, b);
  if (tile * at_once >= s.n * p.G) return;
  Run run;
  if (!PACKED) columns = columns_of(a, tiled);
  if (!find_run(a, columns, 0, b, run) || run.count <= 1 || refused(a, columns, b, s)) return;
  merge_rows<T, D, true>(a, s, run, first_part<true>(a, columns, run), h, tile * at_once, PACKED ? s.n * p.G : merge_tiles * at_once, slices, sm);
}

// The same where the logits of up to 32 rows have been kept: beside the merge of its rows, each workgroup adds all rows'
// probabilities of a piece of the columns to the weights.  The references and sums come from the shares, like the output's.
// grid: pieces of the columns x KV heads x sequences.
template <typename T, int D>
__global__ __launch_bounds__(PA_THREADS) void merge_weigh_kernel(Attend a, int pieces, int slices) {
  constexpr int OR = D + 4;
  __shared__ Merged sm;
  __shared__ float2 stat[32];                  // a row's reference and 1 / its sum, as Attend::stat has them
  const Pages& p = a.p;
  const int piece = (int)(blockIdx.x % pieces), rest = (int)(blockIdx.x / pieces), h = rest % p.Hkv, b = rest / p.Hkv, tid = threadIdx.x;
  const Seq s = load_seq(p, a.starts, a.tokens, a.longest, b);
  const int rows = s.n * p.G, c0 = piece * (4 * PA_THREADS);
  const int at_once = MERGE_ROWS<D> / slices;
  if (rows < a.least_rows || rows > a.most_rows || (c0 >= s.len && piece * at_once >= rows)) return;
  Run run;
  const Columns columns = columns_of(a, false);
  if (!find_run(a, columns, 0, b, run) || refused(a, columns, b, s)) return;
  const int part0 = first_part<false>(a, columns, run);
  const int c = c0 + 4 * tid;
  const bool mine = c < s.len;
  float4 w = make_float4(0.f, 0.f, 0.f, 0.f);
  float* weights = p.weights + track_row(p, b, h) + c;
  if (mine) w = *reinterpret_cast<const float4*>(weights);
  if (c0 < s.len)
    for (int row = tid >> 4; row < rows; row += 16) {          // 16 lanes a row, each with every 16th share
      float M = REF_NONE, L = 0.f;
      const size_t far = (size_t)p.Hkv * a.tiles * a.rows * OR;
      const float* part = a.part + (((size_t)part0 * p.Hkv + h) * a.tiles * a.rows + row) * OR + D;
      for (int z = tid & 15; z < run.count; z += 16) {
        const float2 ml = *reinterpret_cast<const float2*>(part + z * far);
        const float to = fmaxf(M, ml.x);
        L = L * fast_exp2(M - to) + ml.y * fast_exp2(ml.x - to);
        M = to;
      }
#pragma unroll
      for (int x = 1; x <= 8; x <<= 1) {
        const float M2 = __shfl_xor(M, x, 64), L2 = __shfl_xor(L, x, 64), to = fmaxf(M, M2);
        L = L * fast_exp2(M - to) + L2 * fast_exp2(M2 - to);
        M = to;
      }
      if ((tid & 15) == 0) stat[row] = stat_of_sums(M, L);
    }
  __syncthreads();
  if (mine) {
    const float* x = a.logits + ((size_t)b * p.Hkv + h) * a.rows * p.cap + c;
    float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int row = 0; row < rows; ++row) {
      const float4 y = *reinterpret_cast<const float4*>(x + (size_t)row * p.cap);
      const float2 l = stat[row];
      // (a NaN adds nothing)
      f.x = fmaf(fmaxf(fast_exp2(y.x - l.x), 0.f), l.y, f.x); f.y = fmaf(fmaxf(fast_exp2(y.y - l.x), 0.f), l.y, f.y);
      f.z = fmaf(fmaxf(fast_exp2(y.z - l.x), 0.f), l.y, f.z); f.w = fmaf(fmaxf(fast_exp2(y.w - l.x), 0.f), l.y, f.w);
    }
    w.x += f.x; w.y += f.y; w.z += f.z; w.w += f.w;          // (once: a weight is large beside what it gains)
    if (c + 4 <= s.len) *reinterpret_cast<float4*>(weights) = w;
    else {
      const float z[4] = {w.x, w.y, w.z, w.w};
      for (int i = 0; i < s.len - c; ++i) weights[i] = z[i];
    }
  }
  if (run.count > 1) merge_rows<T, D, false>(a, s, run, part0, h, piece * at_once, pieces * at_once, slices, sm);
}

// ---- weights -----------------------------------------------------------------------------------
// A wave takes two blocks of columns and goes through the rows that see them.  grid: column tiles x KV heads x sequences.
template <typename T, int D>
__global__ __launch_bounds__(PA_THREADS, 2) void weigh_kernel(Attend a, int col_tiles) {
  using O = Ops<T, D>;
  constexpr int BK = O::COLS / 16, COLS = O::COLS, ROWB = D * (int)sizeof(T), NB = 2, WIDE = NB * COLS;
  const Pages& p = a.p;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, q4 = lane >> 4;
  const int ct = (int)(blockIdx.x % col_tiles), rest = (int)(blockIdx.x / col_tiles), h = rest % p.Hkv, b = rest / p.Hkv;
  const Seq s = load_seq(p, a.starts, a.tokens, a.longest, b);
  const int c0 = (ct * PA_WAVES + wave) * WIDE;
  if (s.n * p.G < a.least_rows || c0 >= s.len) return;
  if (begins_inside(a.starts, a.tokens, b, s.first)) return;
  const int32_t* table = p.table + (size_t)b * p.width;
  const int in_page = (1 << p.bits) - 1, old = s.len - s.n, rows = s.n * p.G;
  typename O::Keys k[NB];
  bool there[NB][BK];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int x = 0; x < BK; ++x) {
      const int c = c0 + nb * COLS + 16 * x, page = c < s.len ? table[c >> p.bits] : -1;
      there[nb][x] = page >= 0 && page < p.pages;
      const size_t at = ((((size_t)(there[nb][x] ? page : 0) * p.Hkv + h) << p.bits) + (c & in_page)) * ROWB;
      O::load_k(k[nb], x, p.k + at, r * ROWB + q4 * 16);
    }
  float acc[NB][O::NCOL] = {};
  const int first = max(0, c0 - old) * p.G / 16 * 16;       // rows before see none of the columns
#pragma unroll 1
  for (int row0 = first; row0 < rows; row0 += 16) {
    const int row = min(row0 + r, rows - 1), i = row / p.G, head = h * p.G + row - i * p.G;
    const int see = row0 + r < rows ? old + i + 1 : 0;
    const float2 to = a.stat[(size_t)(s.first + i) * p.H + head];
    typename O::Query q;
    O::load_q(q, reinterpret_cast<const T*>(a.q + (s.first + i) * a.q_far) + (size_t)head * D, q4);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      typename O::Logits x;
      logits<D>(x, k[nb], q);
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) {
        const float logit = O::at(x, j) * a.scale_log2e, y = fmaxf(fast_exp2(logit - to.x), 0.f);       // (of a NaN 0)
        acc[nb][j] += c0 + nb * COLS + O::col(q4, j) < see ? y * to.y : 0.f;
      }
    }
  }
  float* weights = p.weights + track_row(p, b, h);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int j = 0; j < O::NCOL; ++j) {
      const float y = group_sum<16>(acc[nb][j]);
      const int c = c0 + nb * COLS + O::col(q4, j);
      if (r == 0 && there[nb][j * BK / O::NCOL] && c < s.len) weights[c] += y;
    }
}

// ---- many rows, bf16 -----------------------------------------------------------------------------
// 32 rows a wave, four waves a workgroup; K and V pass through LDS in tiles of 64 columns, copied a tile ahead (one barrier a
// tile).  32x32x16 products: S^T = K Q^T, where a lane has row l % 32 and, of each half of the tile, columns
// 8 (i/4) + 4 (l/32) + i % 4.  Those are its columns of the B operand of O^T += V^T P^T too (a sum does not ask for the order of
// its terms); the A operand takes the same columns of a dimension out of LDS by two transposing reads.  A row's 16-byte pieces are
// stored under their number XOR one of the row, so that the lanes of a read meet all banks.
// A tile is as much vector work (exponentials at a quarter of the rate, 26 cycles a logit and lane) as matrix work (32 cycles a
// product), and a wave issues in order: the logits of the next tile are formed beside the exponentials of this one, the second
// products beside the rest of them and the next maxima, interleaved by hand step by step.
constexpr int TILED_SUB = TILE / PA_WAVES;                 // a wave copies the 16 columns of one page
template <int D> __device__ inline int swap_k(int row) { return row & (D / 8 - 1); }
template <int D> __device__ inline int swap_v(int row) { return (row & (D / 16 - 1)) << 1; }

typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4s_t lds_v4s_t;
__device__ inline uint2 read_turned(const char* p) {
  return __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4s_t*)(lds_void_t*)p));
}
__device__ inline float other_half(float v) { return __shfl_xor(v, 32, 64); }
// async_copy16 from a uniform base and a lane's offset.
__device__ inline void async_copy16_at(const char* base, unsigned offset, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(offset), "s"(base), "s"(lds_base) : "memory");
}

// An exponential's argument is one multiply-add, logit * scale - reference, which is off by what the reference was rounded by.  Past
// this size that would tell (from 2^31 on it can be 2^7), and the logit is rounded before it like the reference.
constexpr float LARGE = 1 << 20;

template <int D>
__global__ __launch_bounds__(PA_THREADS, 2) void attend_tiled_kernel(Attend a) {
  constexpr int KS = D / 16, DB = D / 32, ROWB = D * 2, HALF = TILE * ROWB, OR = D + 4;
  constexpr int PIECES = D / 8, AT_ONCE = 64 / PIECES, COPIES = TILED_SUB / AT_ONCE;    // rows a copy instruction brings
  extern __shared__ __attribute__((aligned(1024))) char pt_smem[];      // two stages of K, then of V
  const Pages& p = a.p;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, hf = lane >> 5;
  const Place place = place_of(p.Hkv, a.shares, a.tiles);        // the longest tiles first
  if (place.tile >= a.tiles) return;
  const int tile = a.tiles - 1 - place.tile, h = place.group % p.Hkv, w = place.group / p.Hkv;
  const Columns columns = columns_of(a, true);
  if (blockIdx.x == 0 && a.status) write_status(p, a.starts, a.tokens, a.longest, columns.odd, a.status, PA_THREADS);
  const int size = columns.size;
  Run run;
  if (!find_run(a, columns, w, -1, run)) return;
  const Seq s = load_seq(p, a.starts, a.tokens, a.longest, run.b);
  const int rows = s.n * p.G, row0 = tile * TILED_ROWS;
  if (row0 >= rows || refused(a, columns, run.b, s)) return;
  const int old = s.len - s.n, part0 = first_part<true>(a, columns, run) + part_at(a.sparse, w - run.first);
  const int all_see = old + row0 / p.G + 1, end = old + (min(row0 + TILED_ROWS, rows) - 1) / p.G + 1;
  const int lo = (w - run.first) * size, hi = min(lo + size, end);
  // logits are compared before they are scaled, so the scale's sign goes to the queries
  const float scale = fabsf(a.scale_log2e);
  const int row = row0 + wave * 32 + r, at_row = min(row, rows - 1), token = at_row / p.G, head = h * p.G + at_row - token * p.G;
  const int see = min(old + token + 1, hi);
  uint4 q[KS];
  {
    const char* src = a.q + (s.first + token) * a.q_far + (size_t)head * ROWB + hf * 16;
    const unsigned flip = a.scale_log2e < 0.f ? 0x80008000u : 0u;
#pragma unroll
    for (int x = 0; x < KS; ++x) {
      const uint4 u = *reinterpret_cast<const uint4*>(src + x * 32);
      q[x] = make_uint4(u.x ^ flip, u.y ^ flip, u.z ^ flip, u.w ^ flip);
    }
  }
  f32x16_t o[DB] = {};
  float ref = REF_NONE, sum = 0.f, mx = -INFINITY;
  bool large = false;                                  // a reference of the wave is
  const int32_t* table = p.table + (size_t)run.b * p.width;
  const int in_page = (1 << p.bits) - 1;
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(pt_smem)) + wave * TILED_SUB * ROWB;
  unsigned from_k[COPIES], from_v[COPIES];
#pragma unroll
  for (int j = 0; j < COPIES; ++j) {
    const int x = j * AT_ONCE + lane / PIECES, piece = lane % PIECES;
    from_k[j] = x * ROWB + ((piece ^ swap_k<D>(x)) << 4);
    from_v[j] = x * ROWB + ((piece ^ swap_v<D>(x)) << 4);
  }
  // The pages of 16 tiles at a time, a quarter of a tile to a lane, the next ones already asked for: a lookup per tile would be
  // waited for every time (with it, and nothing else to wait for, a tile took 5600 cycles of which 2048 are products).
  const int tiles = (hi - lo + TILE - 1) / TILE;
  auto look_up = [&](int window) {
    const int c = lo + (window * 64 + lane) * TILED_SUB;
    const int page = c < hi ? table[c >> p.bits] : -1;
    return page >= 0 && page < p.pages ? page : -1;
  };
  int window = 0, page0 = lo < hi ? look_up(0) : -1, page1 = lo < hi ? look_up(1) : -1;
  unsigned long long is0 = __ballot(page0 >= 0), is1 = __ballot(page1 >= 0);
  // which quarters of tile t are there
  auto quarters = [&](int t) { return (unsigned)((t >> 4 == window ? is0 : is1) >> (4 * (t & 15))) & 15u; };
  // this wave's quarter of tile t on its way into a stage (of nobody's: any rows)
  auto request = [&](const char* pool, const unsigned (&from)[COPIES], int t, unsigned to) {
    const int at = 4 * (t & 15) + wave, page = t >> 4 == window ? __builtin_amdgcn_readlane(page0, at) : __builtin_amdgcn_readlane(page1, at);
    const char* base = pool + ((((size_t)max(page, 0) * p.Hkv + h) << p.bits) + ((lo + t * TILE + TILED_SUB * wave) & in_page)) * ROWB;
#pragma unroll
    for (int j = 0; j < COPIES; ++j) async_copy16_at(base, from[j], lds0 + to + j * 1024);
  };
  // the reads of a tile's keys, and of its values turned: piece 4 e + .. of rows .. + 4 hf, 8 bytes a lane
  const unsigned at_k = r * ROWB + ((hf ^ swap_k<D>(r)) << 4);                            // of step y: XOR 2 y pieces
  const int turned_row = 4 * hf + ((lane & 15) >> 2);
  const unsigned at_v = turned_row * ROWB + ((((lane >> 4) & 1) * 2 + ((lane & 3) >> 1) ^ swap_v<D>(turned_row)) << 4) + (lane & 1) * 8;   // of e: XOR 4 e pieces
  static_assert(8 % (D / 16) == 0 && 32 % (D / 8) == 0, "the rows of the other reads, 8 and 32 further on, are swapped alike");

  f32x16_t x[2];
  auto mask = [&](int c0, unsigned there) {
    int last = see - c0 - 4 * hf;
    asm volatile("" : "+v"(last));                   // (keeps the comparisons out of the tiles that need none)
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int c = z * 32 + 8 * (i >> 2) + (i & 3);
        if (!(there >> (c / TILED_SUB) & 1) || c >= last) x[z][i] = -INFINITY;
      }
  };
  auto largest = [&]() {
    float m = x[0][0];
#pragma unroll
    for (int i = 1; i < 32; ++i) m = fmaxf(m, x[i >> 4][i & 15]);
    mx = m * scale;
  };

  unsigned now = 0;
  if (lo < hi) {
    now = quarters(0);
    request(p.k, from_k, 0, 0);
    request(p.k, from_k, 1, HALF);
    request(p.v, from_v, 0, 2 * HALF);
    wait_vmcnt<2 * COPIES>();
    __syncthreads();
    x[0] = x[1] = f32x16_t{};
#pragma unroll
    for (int y = 0; y < KS; ++y)
#pragma unroll
      for (int z = 0; z < 2; ++z) x[z] = mfma_wide(*reinterpret_cast<const uint4*>(pt_smem + z * 32 * ROWB + (at_k ^ (y << 5))), q[y], x[z]);
    if (now != (1u << PA_WAVES) - 1 || lo + TILE > all_see) mask(lo, now);
    largest();
  }
  int here = 0;                                        // this tile's stage (its keys are no longer needed)
#pragma unroll 1
  for (int t = 0; t < tiles; ++t) {
    const int c0 = lo + t * TILE;
    // the keys of the next tile and the values of this one are there, and nobody reads those of the last one any more
    wait_vmcnt<0>();
    __syncthreads();
    if (t >> 4 != window) {
      ++window;
      page0 = page1;
      is0 = is1;
      page1 = look_up(window + 1);
      is1 = __ballot(page1 >= 0);
    }
    const unsigned next = quarters(t + 1);
    request(p.k, from_k, t + 2, here);
    request(p.v, from_v, t + 1, 2 * HALF + (HALF - here));
    const char* k = pt_smem + (HALF - here);
    char* v = pt_smem + 2 * HALF + here;
    const bool whole = now == (1u << PA_WAVES) - 1 && c0 + TILE <= all_see;
    bool odd = false;
    if (!whole) {
      // rows of nobody become 0; what is not finite is taken out, and added below for the rows that attend it
      bool mine = false;
#pragma unroll
      for (int y = 0; y < TILED_SUB * (D / 8) / 64; ++y) {
        const int n = y * 64 + lane, vr = wave * TILED_SUB + n / (D / 8);
        uint4* at = reinterpret_cast<uint4*>(v + vr * ROWB + (n % (D / 8) << 4));
        uint4 u = *at;
        if (!(now >> wave & 1) || c0 + vr >= hi) u = make_uint4(0, 0, 0, 0);
        const unsigned f = finite_halves(u.x) & finite_halves(u.y) & finite_halves(u.z) & finite_halves(u.w) & 0x80008000u;
        mine |= f != 0x80008000u;
        *at = make_uint4(keep_finite(u.x), keep_finite(u.y), keep_finite(u.z), keep_finite(u.w));
      }
      odd = __syncthreads_or(mine);
    }
    if (__any(mx > ref + 8.f)) {
      const float top = fmaxf(mx, other_half(mx));
      const float to = top > ref + 8.f ? top : ref, f = fast_exp2(ref - to);
      sum *= f;
#pragma unroll
      for (int e = 0; e < DB; ++e) o[e] *= f;
      ref = to;
      large = __any(fabsf(ref) > LARGE);
    }
    float by = scale;
    if (large) {
#pragma unroll
      for (int i = 0; i < 32; ++i) x[i >> 4][i & 15] *= scale;
      by = 1.f;
    }
    // Probabilities of this tile beside the logits of the next (of what is behind the last one: not used), 16 columns of all rows
    // after the other; three of these four groups beside the first products.  A step forms some exponentials, the arguments of the
    // next step's, and takes in those of the last step; operands are read AHEAD steps before.
    constexpr int STEPS = 2 * KS, VSTEPS = 4 * DB, GROUP = 8, ALL = 4 * GROUP, AHEAD = 2;
    f32x16_t n[2] = {};
    uint4 kf[AHEAD + 1], vf[AHEAD + 1];
    float arg[ALL], e[ALL];
    unsigned pr[16];
    auto read_k = [&](int y) { return *reinterpret_cast<const uint4*>(k + (y & 1) * 32 * ROWB + (at_k ^ (y >> 1 << 5))); };
    auto read_v = [&](int y) {
      const char* src = v + y / DB * 16 * ROWB + (at_v ^ (y % DB << 6));
      const uint2 u0 = read_turned(src), u1 = read_turned(src + 8 * ROWB);
      return make_uint4(u0.x, u0.y, u1.x, u1.y);
    };
    auto argument = [&](int i) { const int g = i / GROUP; arg[i] = fmaf(x[g >> 1][8 * (g & 1) + i % 8], by, -ref); };
    auto take = [&](int i) {
      const int g = i / GROUP;
      sum += e[i];
      if (i & 1) pr[4 * g + i % 8 / 2] = narrow2(e[i - 1], e[i]);
    };
    auto first_of = [&](int y) { return y < STEPS ? y * (3 * GROUP) / STEPS : min(ALL, 3 * GROUP + (y - STEPS) * GROUP / (VSTEPS / 2)); };
#pragma unroll
    for (int y = 0; y < AHEAD; ++y) kf[y] = read_k(y);
#pragma unroll
    for (int i = 0; i < first_of(1); ++i) argument(i);
#pragma unroll
    for (int y = 0; y < STEPS; ++y) {
      if (y + AHEAD < STEPS) kf[(y + AHEAD) % (AHEAD + 1)] = read_k(y + AHEAD);
      else vf[y + AHEAD - STEPS] = read_v(y + AHEAD - STEPS);
      n[y & 1] = mfma_wide(kf[y % (AHEAD + 1)], q[y >> 1], n[y & 1]);
#pragma unroll
      for (int i = first_of(y); i < first_of(y + 1); ++i) e[i] = fast_exp2(arg[i]);
#pragma unroll
      for (int i = first_of(y + 1); i < first_of(y + 2); ++i) argument(i);
      if (y > 0)
#pragma unroll
        for (int i = first_of(y - 1); i < first_of(y); ++i) take(i);
      __builtin_amdgcn_sched_barrier(0);
    }
    float m = n[0][0];
#pragma unroll
    for (int z = 0; z < VSTEPS; ++z) {
      const int y = STEPS + z, g = z / DB;
      if (z + AHEAD < VSTEPS) vf[(z + AHEAD) % (AHEAD + 1)] = read_v(z + AHEAD);
      o[z % DB] = mfma_wide(vf[z % (AHEAD + 1)], make_uint4(pr[4 * g], pr[4 * g + 1], pr[4 * g + 2], pr[4 * g + 3]), o[z % DB]);
#pragma unroll
      for (int i = first_of(y - 1); i < first_of(y); ++i) take(i);
#pragma unroll
      for (int i = first_of(y); i < first_of(y + 1); ++i) e[i] = fast_exp2(arg[i]);
#pragma unroll
      for (int i = first_of(y + 1); i < first_of(y + 2); ++i) argument(i);
      if (z >= VSTEPS / 2) {
        const int u = z - VSTEPS / 2;
#pragma unroll
        for (int i = u * 64 / VSTEPS; i < (u + 1) * 64 / VSTEPS; ++i) m = fmaxf(m, n[i >> 4][i & 15]);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    x[0] = n[0];
    x[1] = n[1];
    mx = m * scale;
    if (next != (1u << PA_WAVES) - 1 || c0 + 2 * TILE > all_see) {
      mask(c0 + TILE, next);
      largest();
    }
    if (odd) {
#pragma unroll 1
      for (int c = c0; c < min(c0 + TILE, hi); ++c) {
        if (!(now >> ((c - c0) / TILED_SUB) & 1)) continue;
        const char* src = p.v + ((((size_t)table[c >> p.bits] * p.Hkv + h) << p.bits) + (c & in_page)) * ROWB + hf * 8;
#pragma unroll
        for (int f = 0; f < DB; ++f)
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const uint2 u = *reinterpret_cast<const uint2*>(src + (32 * f + 8 * z) * 2);
            const unsigned word[4] = {u.x << 16, u.x & 0xffff0000u, u.y << 16, u.y & 0xffff0000u};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float bad = __uint_as_float(word[i] & ~(unsigned)((int)finite_word(word[i]) >> 31));
              o[f][4 * z + i] += c < see ? bad : 0.f;
            }
          }
      }
    }
    now = next;
    here = HALF - here;
  }
  wait_vmcnt<0>();                                     // (copies into LDS that nobody waits for)
  const float total = sum + other_half(sum);
  if (row >= rows) return;
  float* part = a.part + (((size_t)part0 * p.Hkv + h) * a.tiles * TILED_ROWS + row) * OR;
  const size_t at = (size_t)(s.first + token) * p.H + head;
  const bool any = !(total == 0.f);
  const float inv = any ? 1.0f / total : 0.f;
#pragma unroll
  for (int f = 0; f < DB; ++f)
#pragma unroll
    for (int z = 0; z < 4; ++z) {
      const int c = 32 * f + 8 * z + 4 * hf;
      const float4 u = make_float4(o[f][4 * z], o[f][4 * z + 1], o[f][4 * z + 2], o[f][4 * z + 3]);
      if (run.count > 1) *reinterpret_cast<float4*>(part + c) = u;
      else store4(a.out, at * D + c, any ? u : make_float4(0.f, 0.f, 0.f, 0.f), inv, uint16_t());
    }
  if (hf == 0) {
    if (run.count > 1) *reinterpret_cast<float2*>(part + D) = make_float2(ref, total);
    else finish_sums(a, at, ref, total);
  }
}

// Weights of many rows: 32 columns a wave, their keys in registers; the rows' queries pass through LDS in tiles of 64.  A lane
// has row l % 32 and adds up its columns over the rows it meets; the lanes are added at the end.  grid: column tiles x KV heads x
// sequences.
template <int D>
__global__ __launch_bounds__(PA_THREADS, 3) void weigh_tiled_kernel(Attend a, int col_tiles, int splits) {
  constexpr int KS = D / 16, ROWB = D * 2, STAGE = TILE * ROWB;
  constexpr int PIECES = D / 8, AT_ONCE = 64 / PIECES, COPIES = TILED_SUB / AT_ONCE;
  extern __shared__ __attribute__((aligned(1024))) char pt_smem[];      // two stages of queries
  const Pages& p = a.p;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 31, hf = lane >> 5;
  const Place place = place_of(p.Hkv, p.B, col_tiles * splits);
  const int ct = place.tile % col_tiles, split = place.tile / col_tiles, h = place.group % p.Hkv, b = place.group / p.Hkv;
  if (split >= splits || b >= p.B) return;
  const Seq s = load_seq(p, a.starts, a.tokens, a.longest, b);
  const int first_col = ct * (PA_WAVES * 32), c0 = first_col + wave * 32;
  if (s.n * p.G < a.least_rows || first_col >= s.len) return;
  if (begins_inside(a.starts, a.tokens, b, s.first)) return;
  const int32_t* table = p.table + (size_t)b * p.width;
  const int in_page = (1 << p.bits) - 1, old = s.len - s.n;
  uint4 k[KS];
  {
    const int c = c0 + r, page = c < s.len ? table[c >> p.bits] : -1;
    const size_t at = ((((size_t)(page >= 0 && page < p.pages ? page : 0) * p.Hkv + h) << p.bits) + (c & in_page)) * ROWB + hf * 16;
#pragma unroll
    for (int y = 0; y < KS; ++y) k[y] = *reinterpret_cast<const uint4*>(p.k + at + y * 32);
  }
  const unsigned lds0 = __builtin_amdgcn_readfirstlane(lds_address(pt_smem)) + wave * TILED_SUB * ROWB;
  // A tile holds whole tokens, so that its rows lie the same way from its first token on: their places are worked out once.
  const int per = TILE / p.G;                          // tokens
  const char* q0 = a.q + s.first * a.q_far + (size_t)h * p.G * ROWB;
  const float2* stat0 = a.stat + (size_t)s.first * p.H + h * p.G;
  int token_of[COPIES];
  unsigned from[COPIES];                               // the piece of its row, without the token
#pragma unroll
  for (int j = 0; j < COPIES; ++j) {
    const int x = j * AT_ONCE + lane / PIECES, row = wave * TILED_SUB + x;
    token_of[j] = min(row / p.G, per - 1);             // (behind the tile's rows: any)
    from[j] = row % p.G * ROWB + (((lane % PIECES) ^ swap_k<D>(x)) << 4);
  }
  auto request = [&](int first, int stage) {
    const char* base = q0 + first * a.q_far;
    const int last = s.n - 1 - first;
#pragma unroll
    for (int j = 0; j < COPIES; ++j)
      async_copy16_at(base, (unsigned)min(token_of[j], last) * (unsigned)a.q_far + from[j], lds0 + stage * STAGE + j * 1024);
  };
  int my_token[2], my_stat[2];
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int row = 32 * y + r;
    my_token[y] = row / p.G < per ? row / p.G : s.n;   // (behind the tile's rows: no token)
    my_stat[y] = min(row / p.G, per - 1) * p.H + row % p.G;
  }
  float2 l[2];
  int see[2];
  auto stats = [&](int first) {                        // rows of no token: exponentials of minus infinity
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const bool in = my_token[y] < s.n - first;
      const float2 u = stat0[(size_t)first * p.H + (in ? my_stat[y] : 0)];
      l[y] = in ? u : make_float2(INFINITY, 0.f);
      see[y] = old + first + my_token[y] + 1 - c0;
    }
  };
  f32x16_t acc = {};
  const int sees_it = max(0, first_col - old);         // tokens before see none of the columns
  const int share = ((s.n - sees_it + per - 1) / per + splits - 1) / splits * per;
  const int begin = min(sees_it + split * share, s.n), end = min(begin + share, s.n);
  if (begin < end) {
    request(begin, 0);
    stats(begin);
  }
  int stage = 0;
  const unsigned at_q = r * ROWB + ((hf ^ swap_k<D>(r)) << 4);        // of step e: XOR 2 e pieces
  struct Yes { __device__ constexpr operator bool() const { return true; } };
  struct No { __device__ constexpr operator bool() const { return false; } };
  auto tile = [&](const char* q, const float2 (&now)[2], const int (&sees)[2], auto masked) {
    unsigned from = at_q;
    float scale = a.scale_log2e;
    asm volatile("" : "+v"(from), "+v"(scale));       // (or what both forms of a tile share is worked out, and held, before the choice)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      f32x16_t x = {};
#pragma unroll
      for (int e = 0; e < KS; ++e) x = mfma_wide(k[e], *reinterpret_cast<const uint4*>(q + y * 32 * ROWB + (from ^ (e << 5))), x);
      float by = scale;
      if (__any(fabsf(now[y].x) > LARGE && now[y].y > 0.f)) {
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] *= scale;
        by = 1.f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float e = fmaxf(fast_exp2(fmaf(x[i], by, -now[y].x)), 0.f);        // (of a NaN 0)
        if (masked && 8 * (i >> 2) + 4 * hf + (i & 3) >= sees[y]) e = 0.f;
        acc[i] = fmaf(e, now[y].y, acc[i]);
      }
    }
  };
#pragma unroll 1
  for (int first = begin; first < end; first += per, stage ^= 1) {
    wait_vmcnt<0>();
    __syncthreads();
    const float2 now[2] = {l[0], l[1]};
    const int sees[2] = {see[0], see[1]};
    if (first + per < end) {
      request(first + per, stage ^ 1);
      stats(first + per);
    }
    const char* q = pt_smem + stage * STAGE;
    if (old + first + 1 >= c0 + 32) tile(q, now, sees, No());
    else tile(q, now, sees, Yes());
  }
  float* weights = p.weights + track_row(p, b, h);
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const float e = group_sum<32>(acc[i]);
    const int c = c0 + 8 * (i >> 2) + 4 * hf + (i & 3);
    if (r == 0 && c < s.len) {
      const int page = table[c >> p.bits];
      if (splits > 1) a.gains[(((size_t)split * p.B + b) * p.Hkv + h) * p.cap + c] = e;
      else if (page >= 0 && page < p.pages) weights[c] += e;
    }
  }
}

// The splits' sums go to the weights.  grid: pieces of the columns x KV heads x sequences.
__global__ __launch_bounds__(PA_THREADS) void add_gains_kernel(Attend a, int pieces, int splits) {
  const Pages& p = a.p;
  const int c = (int)(blockIdx.x % pieces) * PA_THREADS + threadIdx.x, rest = (int)(blockIdx.x / pieces), h = rest % p.Hkv, b = rest / p.Hkv;
  const Seq s = load_seq(p, a.starts, a.tokens, a.longest, b);
  const bool inside = begins_inside(a.starts, a.tokens, b, s.first);
  if (s.n * p.G < a.least_rows || c >= s.len || inside) return;
  const int page = p.table[(size_t)b * p.width + (c >> p.bits)];
  if (page < 0 || page >= p.pages) return;
  const float* gain = a.gains + ((size_t)b * p.Hkv + h) * p.cap + c;
  const size_t far = (size_t)p.B * p.Hkv * p.cap;
  float e = 0.f;
  for (int z = 0; z < splits; ++z) e += gain[z * far];
  p.weights[track_row(p, b, h) + c] += e;
}

// ---- launches ----------------------------------------------------------------------------------
// Groups of threads for a row's shares: each takes up to eight, all on their way together (one token behind 8000, 8 KV heads, 32
// shares: 33.6 us with one group, 16.5 with four).
template <int D>
int merge_slices(const Attend& a) {
  int slices = 1;
  while (slices < MERGE_ROWS<D> && (a.shares / a.p.B + 1) > 8 * slices) slices *= 2;
  return slices;
}
// The attention of the sequences with least_rows to most_rows rows.
template <typename T, int D>
int launch_shares(const Attend& a, bool tiled, bool keep, hipStream_t s) {
  constexpr int OR = D + 4;
  const Pages& p = a.p;
  // shares: where they are of one sequence each, one more for each sequence but one at most
  const unsigned groups = (unsigned)(a.shares + p.B - 1) * p.Hkv;
  if (tiled) {
    if constexpr (sizeof(T) == 2) {
      const int lds = 4 * TILE * D * 2;
      auto kernel = attend_tiled_kernel<D>;
      if (lds > 48 * 1024 && hip_failed(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds))) return TREEKV_EHIP;
      hipLaunchKernelGGL(kernel, dim3(places(groups, p.Hkv, a.shares, a.tiles)), dim3(PA_THREADS), lds, s, a);
    }
  } else {
    const size_t lds = (size_t)PA_WAVES * a.rows * (OR * 4 + 8);
    auto kernel = a.rows != 16 ? keep ? attend_kernel<T, D, 2, true> : attend_kernel<T, D, 2, false> : keep ? attend_kernel<T, D, 1, true> : attend_kernel<T, D, 1, false>;
    if (lds > 48 * 1024 && hip_failed(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds))) return TREEKV_EHIP;
    hipLaunchKernelGGL(kernel, dim3(groups * a.tiles), dim3(PA_THREADS), lds, s, a);
  }
  if (a.shares > 1 && !keep) {
    const int slices = merge_slices<D>(a), at_once = MERGE_ROWS<D> / slices;
    const MergeGrid m = merge_grid(p.B, p.Hkv, p.G, a.tokens, std::min(a.longest * p.G, a.most_rows), at_once);
    if (m.packed) hipLaunchKernelGGL((merge_kernel<T, D, true>), dim3((unsigned)p.Hkv * m.groups), dim3(PA_THREADS), 0, s, a, m.groups, slices, tiled);
    else hipLaunchKernelGGL((merge_kernel<T, D, false>), dim3((unsigned)(p.Hkv * p.B) * m.groups), dim3(PA_THREADS), 0, s, a, m.groups, slices, tiled);
  }
  return finish_launch();
}

// What they add to the weights, and the merge, where the logits have been kept.
template <typename T, int D>
int launch_kept(const Attend& a, hipStream_t s) {
  const Pages& p = a.p;
  const int slices = merge_slices<D>(a), at_once = MERGE_ROWS<D> / slices;
  const int all = std::max((p.cap + 4 * PA_THREADS - 1) / (4 * PA_THREADS), (std::min(a.longest * p.G, a.most_rows) + at_once - 1) / at_once);
  hipLaunchKernelGGL((merge_weigh_kernel<T, D>), dim3((unsigned)(p.Hkv * p.B) * all), dim3(PA_THREADS), 0, s, a, all, slices);
  return finish_launch();
}

template <typename T, int D>
int launch_attend_d(Attend a, const AttendShape& sh, int weigh, hipStream_t s) {
  const Pages& p = a.p;
  if (sh.short_shares) {
    Attend few = a;
    few.part = (float*)((char*)a.part + sh.part);
    few.tiles = 1; few.rows = 16; few.shares = sh.short_shares;
    few.most_rows = 16;
    few.sparse = is_sparse(few.shares, p.B, sh.short_keep);
    if (int e = launch_shares<T, D>(few, false, sh.short_keep, s)) return e;
    if (sh.short_keep)
      if (int e = launch_kept<T, D>(few, s)) return e;
    a.least_rows = 17;
  }
  if (int e = launch_shares<T, D>(a, sh.tiled, sh.keep, s)) return e;
  if (sh.keep) return launch_kept<T, D>(a, s);
  const unsigned units = (unsigned)(p.Hkv * p.B);
  if (weigh) {
    if (!sh.short_keep) a.least_rows = 1;
    if (sh.weigh_tiled && a.q_far < 1 << 24) {         // (places of 64 rows in 32 bits)
      if constexpr (sizeof(T) == 2) {
        const int all = (p.cap + PA_WAVES * 32 - 1) / (PA_WAVES * 32);
        hipLaunchKernelGGL((weigh_tiled_kernel<D>), dim3(places(units, p.Hkv, p.B, all * sh.weigh_splits)), dim3(PA_THREADS), 2 * TILE * D * 2, s, a, all,
                           sh.weigh_splits);
        if (sh.weigh_splits > 1) {
          const int pieces = (p.cap + PA_THREADS - 1) / PA_THREADS;
          hipLaunchKernelGGL(add_gains_kernel, dim3(units * pieces), dim3(PA_THREADS), 0, s, a, pieces, sh.weigh_splits);
        }
      }
    } else {
      constexpr int WIDE = PA_WAVES * 2 * Ops<T, D>::COLS;
      const int all = (p.cap + WIDE - 1) / WIDE;
      hipLaunchKernelGGL((weigh_kernel<T, D>), dim3(units * all), dim3(PA_THREADS), 0, s, a, all);
    }
  }
  return finish_launch();
}

}  // namespace

int launch_paged_append(const treekv_paged_cache& c, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                        const int32_t* starts, int tokens, const int32_t* positions, int32_t* status, hipStream_t s) {
  const int esz = c.dtype == TREEKV_F32 ? 4 : 2, piece_bits = __builtin_ctz(c.head_dim * esz / 16);
  const Pages p = pages_of(c);
  if (tokens <= 2048)
    hipLaunchKernelGGL((append_kernel<1>), dim3(tokens), dim3(PA_THREADS), 0, s, p, (const char*)k, (const char*)v, k_stride * esz,
                       v_stride * esz, starts, tokens, positions, status, piece_bits);
  else
    hipLaunchKernelGGL((append_kernel<16>), dim3((tokens + 15) / 16), dim3(PA_THREADS), 0, s, p, (const char*)k, (const char*)v,
                       k_stride * esz, v_stride * esz, starts, tokens, positions, status, piece_bits);
  return finish_launch();
}

size_t paged_attend_scratch_bytes(const treekv_paged_cache& c, int tokens, int longest, int weigh) {
  const AttendShape s = attend_shape(c, tokens, longest, weigh);
  return s.part + s.short_part + s.logits + s.stat + s.gains;
}

int launch_paged_attend(const treekv_paged_cache& c, const void* q, int64_t q_stride, const int32_t* starts, int tokens, int longest,
                        void* out, float* lse, int weigh, void* scratch, int32_t* status, hipStream_t s) {
  const AttendShape sh = attend_shape(c, tokens, longest, weigh);
  Attend a;
  a.p = pages_of(c);
  a.starts = starts;
  a.q = (const char*)q;
  a.q_far = q_stride * (c.dtype == TREEKV_F32 ? 4 : 2);
  a.out = (char*)out;
  a.part = (float*)scratch;
  a.logits = (float*)((char*)scratch + sh.part + sh.short_part);
  a.stat = sh.stat ? (float2*)((char*)scratch + sh.part + sh.short_part + sh.logits) : nullptr;
  a.gains = (float*)((char*)scratch + sh.part + sh.short_part + sh.logits + sh.stat);
  a.lse = lse;
  a.status = status;
  a.tokens = tokens; a.longest = longest; a.tiles = sh.tiles; a.shares = sh.shares; a.rows = sh.rows;
  a.least_rows = 1; a.most_rows = INT_MAX;
  a.wide = past_32_bits(c);
  a.sparse = is_sparse(sh.shares, c.batch, sh.keep);
  a.scale_log2e = (c.softmax_scale != 0.f ? c.softmax_scale : 1.0f / sqrtf((float)c.head_dim)) * LOG2E;
  if (c.dtype == TREEKV_F32) return c.head_dim == 128 ? launch_attend_d<float, 128>(a, sh, weigh, s) : launch_attend_d<float, 64>(a, sh, weigh, s);
  return c.head_dim == 128 ? launch_attend_d<uint16_t, 128>(a, sh, weigh, s) : launch_attend_d<uint16_t, 64>(a, sh, weigh, s);
}

}  // namespace tkv
