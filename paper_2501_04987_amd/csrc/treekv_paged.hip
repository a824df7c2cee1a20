// A paged cache for gfx950: treekv_paged_append and treekv_paged_attend.
//
// attend   o_i = sum over j <= i of p_ij v_j, p_ij = exp(q_i k_j * scale - lse_i), over a sequence's pages.  The G query heads
//          of a KV head and the sequence's n new tokens are the rows of one matrix product, in tiles of 16 or 32; columns are
//          slots.  A softmax in one pass: the reference of a row's exponentials is raised where a logit passes it by 2^8, sums
//          are fp32.  With bf16 storage P enters the second product rounded to bf16 (2^-9 of each probability at most, where the
//          output is rounded by as much again); the sum beside it takes the unrounded ones.
//          A page holds a multiple of 16 rows, so 16 columns lie in one page: one address for the wave and a lane's offset.
// shares   Few rows leave most of the chip idle, so the columns of the whole batch are cut into equal shares, which the device
//          works out from the lengths: long sequences get more workgroups than short ones.  A sequence's shares are merged by a
//          second kernel.
// weights  the probabilities once more from q, k and lse, summed down the rows: a column belongs to one wave, so the sum needs
//          no atomics and repeats bit for bit.

#include "treekv_matrix.h"
#include "treekv_paged.h"

namespace tkv {

namespace {

constexpr int PA_THREADS = 256, PA_WAVES = PA_THREADS / 64;
constexpr int MIN_SHARE = 128;               // columns: a block for each wave

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
  __shared__ int at_b[TOK], at_slot[TOK], at_page[TOK];
  const int tid = threadIdx.x;
  if (blockIdx.x == 0 && status)
    for (int b = tid; b < p.B; b += PA_THREADS) status[b] = load_seq(p, starts, tokens, tokens, b).ok ? TREEKV_OK : TREEKV_EINVAL;
  const int t0 = (int)blockIdx.x * TOK;
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
  }
  __syncthreads();
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
  int32_t* status;
  int tokens, longest, tiles, shares;        // row tiles of the longest sequence; shares the columns are cut into
  float scale_log2e;
};

// The columns of all sequences with new tokens, cut into pieces of `size`: a sequence's first piece starts at its first
// token.  Piece w is piece `index` of `count` of sequence b, whose first is number `first`.
struct Share {
  int b, index, count, first, size;
};
__device__ inline int tokens_to_read(const Attend& a, int b) {
  if (b >= a.p.B) return 0;
  const Seq s = load_seq(a.p, a.starts, a.tokens, a.longest, b);
  return s.n > 0 ? s.len : 0;
}
__device__ inline int share_size(const Attend& a) {
  long long total = 0;
  for (int b = threadIdx.x & 63; b < a.p.B; b += 64) total += tokens_to_read(a, b);
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) total += __shfl_xor(total, x, 64);
  const long long each = (total + a.shares - 1) / a.shares;
  return (int)max((each + 31) / 32 * 32, (long long)MIN_SHARE);
}
// By piece (want_b < 0) or, its first piece, by sequence.
__device__ inline bool find_share(const Attend& a, int w, int want_b, Share& s) {
  const int lane = threadIdx.x & 63;
  s.size = share_size(a);
  int before = 0;
  for (int b0 = 0; b0 < a.p.B; b0 += 64) {
    const int mine = (tokens_to_read(a, b0 + lane) + s.size - 1) / s.size;
    int sum = mine;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int y = __shfl_up(sum, x, 64);
      if (lane >= x) sum += y;
    }
    const unsigned long long hit = __ballot(want_b < 0 ? before + sum > w : b0 + lane == want_b);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;
      s.b = __builtin_amdgcn_readfirstlane(b0 + l);
      s.count = __builtin_amdgcn_readfirstlane(__shfl(mine, l, 64));
      s.first = __builtin_amdgcn_readfirstlane(before + __shfl(sum, l, 64)) - s.count;
      s.index = w - s.first;
      return true;
    }
    before += __shfl(sum, 63, 64);
  }
  return false;
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
template <typename T, int D>
__device__ inline void finish_row(const Attend& a, const Seq& s, int h, int row, int c, const float4& o, float M, float L) {
  const size_t at = (size_t)(s.first + row / a.p.G) * a.p.H + h * a.p.G + row % a.p.G;
  const bool any = !(L == 0.f);                          // (a sum that is a NaN stays one)
  store4(a.out, at * D + c, any ? o : make_float4(0.f, 0.f, 0.f, 0.f), any ? 1.0f / L : 0.f, T());
  if (c == 0 && a.lse) a.lse[at] = any ? (M + log2f(L)) * LN2 : -INFINITY;
}

// grid: shares of the columns x KV heads x row tiles.  RB: blocks of 16 rows.
template <typename T, int D, int RB>
__global__ __launch_bounds__(PA_THREADS, RB == 1 ? 3 : 2) void attend_kernel(Attend a) {
  using O = Ops<T, D>;
  constexpr int ROWS = RB * 16, DPL = O::DPL, OR = D + 4, BK = O::COLS / 16, COLS = O::COLS, ROWB = D * (int)sizeof(T);
  extern __shared__ __attribute__((aligned(16))) float pa_smem[];
  const Pages& p = a.p;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, r = lane & 15, q4 = lane >> 4;
  const int tile = (int)(blockIdx.x % a.tiles), rest = (int)(blockIdx.x / a.tiles), h = rest % p.Hkv, w = rest / p.Hkv;
  if (blockIdx.x == 0 && a.status)
    for (int b = tid; b < p.B; b += PA_THREADS) a.status[b] = load_seq(p, a.starts, a.tokens, a.longest, b).ok ? TREEKV_OK : TREEKV_EINVAL;
  Share sh;
  if (!find_share(a, w, -1, sh)) return;
  const Seq s = load_seq(p, a.starts, a.tokens, a.longest, sh.b);
  const int rows = s.n * p.G, row0 = tile * ROWS;
  if (row0 >= rows) return;
  const int old = s.len - s.n;
  // columns: what the tile's first row sees all rows see, behind what its last row sees there is nothing for it
  const int all_see = old + row0 / p.G + 1, end = old + (min(row0 + ROWS, rows) - 1) / p.G + 1;
  const int lo = sh.index * sh.size, hi = min(lo + sh.size, end);

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
  const int32_t* table = p.table + (size_t)sh.b * p.width;
  const int in_page = (1 << p.bits) - 1;

#pragma unroll 1
  for (int c0 = lo + wave * COLS; c0 < hi; c0 += PA_WAVES * COLS) {
    size_t at[BK];
    bool there[BK], whole = c0 + COLS <= all_see;
#pragma unroll
    for (int x = 0; x < BK; ++x) {
      const int c = c0 + 16 * x, page = c < hi ? table[c >> p.bits] : -1;
      there[x] = page >= 0 && page < p.pages;
      whole &= there[x];
      at[x] = ((((size_t)(there[x] ? page : 0) * p.Hkv + h) << p.bits) + (c & in_page)) * ROWB;
    }
    typename O::Keys k;
    typename O::Values v;
#pragma unroll
    for (int x = 0; x < BK; ++x) O::load_k(k, x, p.k + at[x], r * ROWB + q4 * 16);
#pragma unroll
    for (int j = 0; j < O::NCOL; ++j) O::load_v(v, j, p.v + at[j * BK / O::NCOL], (O::col(q4, j) & 15) * ROWB + r * DPL * (int)sizeof(T));
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
      typename O::Logits x;
      logits<D>(x, k, q[rb]);
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) {
        float& y = O::at(x, j);
        y *= a.scale_log2e;
        if (!whole && (!there[j * BK / O::NCOL] || c0 + O::col(q4, j) >= min(see[rb], hi))) y = -INFINITY;
        mx = fmaxf(mx, y);
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
    if (sh.count > 1) {
      float* part = a.part + (((size_t)w * p.Hkv + h) * a.tiles + tile) * ROWS * OR + (size_t)y * OR;
      *reinterpret_cast<float4*>(part + c) = f;
      if (c == 0) *reinterpret_cast<float2*>(part + D) = make_float2(M, L);
    } else {
      finish_row<T, D>(a, s, h, row0 + y, c, f, M, L);
    }
  }
}

// Shares of a sequence added.  grid: sequences x KV heads x row tiles.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(PA_THREADS) void merge_kernel(Attend a) {
  constexpr int OR = D + 4;
  const Pages& p = a.p;
  const int tile = (int)(blockIdx.x % a.tiles), rest = (int)(blockIdx.x / a.tiles), h = rest % p.Hkv, b = rest / p.Hkv;
  const Seq s = load_seq(p, a.starts, a.tokens, a.longest, b);
  const int rows = s.n * p.G, row0 = tile * ROWS;
  if (row0 >= rows) return;
  Share sh;
  if (!find_share(a, 0, b, sh) || sh.count <= 1) return;
  for (int x = threadIdx.x; x < ROWS * (D / 4); x += PA_THREADS) {
    const int y = x / (D / 4), c = x % (D / 4) * 4;
    if (row0 + y >= rows) break;
    const size_t far = (size_t)p.Hkv * a.tiles * ROWS * OR;
    const float* part = a.part + (((size_t)sh.first * p.Hkv + h) * a.tiles + tile) * ROWS * OR + (size_t)y * OR;
    float M = REF_NONE, L = 0.f;
    for (int z = 0; z < sh.count; ++z) M = fmaxf(M, part[z * far + D]);
    float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int z = 0; z < sh.count; ++z) {
      const float2 ml = *reinterpret_cast<const float2*>(part + z * far + D);
      const float g = fast_exp2(ml.x - M);
      const float4 u = *reinterpret_cast<const float4*>(part + z * far + c);
      L = fmaf(ml.y, g, L);
      f.x = fmaf(u.x, g, f.x); f.y = fmaf(u.y, g, f.y); f.z = fmaf(u.z, g, f.z); f.w = fmaf(u.w, g, f.w);
    }
    finish_row<T, D>(a, s, h, row0 + y, c, f, M, L);
  }
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
  if (s.n == 0 || c0 >= s.len) return;
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
    const float to = a.lse[(size_t)(s.first + i) * p.H + head] * LOG2E;
    typename O::Query q;
    O::load_q(q, reinterpret_cast<const T*>(a.q + (s.first + i) * a.q_far) + (size_t)head * D, q4);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      typename O::Logits x;
      logits<D>(x, k[nb], q);
#pragma unroll
      for (int j = 0; j < O::NCOL; ++j) {
        const float y = fast_exp2(fmaf(O::at(x, j), a.scale_log2e, -to));
        acc[nb][j] += c0 + nb * COLS + O::col(q4, j) < see && y > 0.f ? y : 0.f;     // (not a NaN)
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

// ---- launches ----------------------------------------------------------------------------------
struct AttendShape {
  int rows, tiles, shares;                   // rows of a tile
  size_t part, lse;                          // bytes of scratch: shares' results, log sums nobody asked for
};
AttendShape attend_shape(const treekv_paged_cache& c, int tokens, int longest, int weigh) {
  const long long rows = (long long)longest * (c.q_heads / c.kv_heads);
  AttendShape s;
  s.rows = rows <= 16 ? 16 : 32;
  s.tiles = (int)((rows + s.rows - 1) / s.rows);
  const long long groups = (long long)c.kv_heads * s.tiles;
  s.shares = (int)(groups >= 768 ? 1 : (768 + groups - 1) / groups);      // three workgroups a compute unit
  const long long cap = (long long)c.table_width * c.page_size, most = ((long long)c.batch * cap + MIN_SHARE - 1) / MIN_SHARE;
  if (s.shares > most) s.shares = (int)most;
  s.part = s.shares > 1 ? align_up((size_t)(s.shares + c.batch) * groups * s.rows * (c.head_dim + 4) * 4) : 0;
  s.lse = weigh ? align_up((size_t)tokens * c.q_heads * 4) : 0;
  return s;
}

template <typename T, int D>
int launch_attend_d(const Attend& a, const AttendShape& sh, int weigh, hipStream_t s) {
  constexpr int OR = D + 4;
  const unsigned groups = (unsigned)(a.p.Hkv * a.tiles);
  const unsigned grid = (unsigned)(a.shares + (a.shares > 1 ? a.p.B : a.p.B - 1)) * groups;
  const size_t lds = (size_t)PA_WAVES * sh.rows * (OR * 4 + 8);
  auto kernel = sh.rows == 16 ? attend_kernel<T, D, 1> : attend_kernel<T, D, 2>;
  if (lds > 48 * 1024 && hip_failed(hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds))) return TREEKV_EHIP;
  hipLaunchKernelGGL(kernel, dim3(grid), dim3(PA_THREADS), lds, s, a);
  if (a.shares > 1) {
    const unsigned all = (unsigned)a.p.B * groups;
    if (sh.rows == 16) hipLaunchKernelGGL((merge_kernel<T, D, 16>), dim3(all), dim3(PA_THREADS), 0, s, a);
    else hipLaunchKernelGGL((merge_kernel<T, D, 32>), dim3(all), dim3(PA_THREADS), 0, s, a);
  }
  if (weigh) {
    constexpr int WIDE = PA_WAVES * 2 * Ops<T, D>::COLS;
    const int col_tiles = (a.p.cap + WIDE - 1) / WIDE;
    hipLaunchKernelGGL((weigh_kernel<T, D>), dim3((unsigned)col_tiles * a.p.Hkv * a.p.B), dim3(PA_THREADS), 0, s, a, col_tiles);
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
  return s.part + s.lse;
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
  a.lse = !lse && weigh ? (float*)((char*)scratch + sh.part) : lse;
  a.status = status;
  a.tokens = tokens; a.longest = longest; a.tiles = sh.tiles; a.shares = sh.shares;
  a.scale_log2e = (c.softmax_scale != 0.f ? c.softmax_scale : 1.0f / sqrtf((float)c.head_dim)) * LOG2E;
  if (c.dtype == TREEKV_F32) return c.head_dim == 128 ? launch_attend_d<float, 128>(a, sh, weigh, s) : launch_attend_d<float, 64>(a, sh, weigh, s);
  return c.head_dim == 128 ? launch_attend_d<uint16_t, 128>(a, sh, weigh, s) : launch_attend_d<uint16_t, 64>(a, sh, weigh, s);
}

}  // namespace tkv
