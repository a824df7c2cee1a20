// Eviction from a paged cache by accumulated weight (treekv_paged_evict) for gfx950.
//
// A unit is one KV head of one sequence.  Of its len tokens the `budget` first by (protected, weight descending, slot) are kept:
//   key     an order-preserving 32-bit image of the weight; protected tokens above all, NaNs as minus infinity
//   choice  the budget-th largest key T, a few bits of it a round, then, in slot order, whatever is above T and the first of what
//           equals it
//   move    attention does not ask for the order of columns, so what is kept stays where it is: only tokens from slots behind
//           the budget move, into the freed slots before it, as many rows as were kept there (of a decode step one, where
//           closing the gaps would move half of the cache)
// Two kernels: one workgroup per unit makes the choice and lists the moves, then all of the chip copies the rows.  32 units of 32768
// slots cut to 4096: the choice takes 27 us in 32 workgroups, of which reading is 10, the threshold 8 and the list of 3350 moves 9, the rows 26
// at 4.2 TB/s in and out (4 where nothing moves); 256 units of 2049 slots 9 and 4, rounds of barriers.  Past 32768 slots keys are
// formed anew in every pass: 8 units of 32768 40 us in all, of 32770 99, of 131072 342.

#include "treekv_paged.h"

namespace tkv {

namespace {

constexpr int EV_THREADS = 1024, EV_WAVES = EV_THREADS / 64, MV_THREADS = 256;

struct Evict {
  Pages p;
  int budget, n_sink, n_recent;
  int2* moves;               // [units][stride] slots: from, to
  int stride;                // most moves of a unit: each needs a slot below the budget and one behind it
  int* count;                // [units] moves; -1: the sequence is left as it is
  int32_t *status, *lens_out;
};

__device__ inline unsigned order_of(float w) {
  if (!(w == w)) w = -INFINITY;
  const unsigned u = __float_as_uint(w == 0.f ? 0.f : w);          // (-0 is 0)
  return u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u);
}

// Sum over the workgroup of a value per wave, for the waves before this one; `total` of all.  Two barriers.
__device__ inline int before_me(int mine, int* sm, int& total) {
  const int wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[wave] = mine;
  __syncthreads();
  int sum = 0;
  total = 0;
  for (int i = 0; i < EV_WAVES; ++i) {
    if (i < wave) sum += sm[i];
    total += sm[i];
  }
  return sum;
}
__device__ inline int below(unsigned long long mask) { return __popcll(mask & ((1ull << (threadIdx.x & 63)) - 1)); }

struct Unit {
  const float* w;
  const int32_t* pos;
  int2* moves;
  int len;
  long long recent;          // positions above it are protected
};
__device__ inline unsigned key_of(const Evict& e, const Unit& u, float w, int pos) {
  return pos < e.n_sink || pos > u.recent ? 0xffffffffu : order_of(w);
}
// Sum, and sums up to each, over 16 consecutive lanes.
template <int CTRL> __device__ inline int dpp_plus(int v) { return v + __builtin_amdgcn_update_dpp(0, v, CTRL, 0xf, 0xf, true); }
__device__ inline int row_sum16(int v) { return dpp_plus<0x121>(dpp_plus<0x122>(dpp_plus<0x124>(dpp_plus<0x128>(v)))); }     // row_ror
__device__ inline int row_scan16(int v) { return dpp_plus<0x118>(dpp_plus<0x114>(dpp_plus<0x112>(dpp_plus<0x111>(v)))); }    // row_shr
__device__ inline int largest_of_all(int mine, int* sm) {
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) mine = max(mine, __shfl_xor(mine, x, 64));
  if ((threadIdx.x & 63) == 0) sm[threadIdx.x >> 6] = mine;
  __syncthreads();
  mine = sm[0];
#pragma unroll
  for (int i = 1; i < EV_WAVES; ++i) mine = max(mine, sm[i]);
  return mine;
}

// T by up to four rounds of 8 bits from the top: a histogram of the keys that agree with T so far, and in it the digit at which
// `budget` is reached.  Weights are of a few orders of magnitude, so in the first round most lanes add to the same bins: COPIES
// histograms beside each other, a bank apart, keep them from waiting for one another.  It ends early where all of a digit's keys
// are kept: then every key at or above T is.
constexpr int COPIES = 16, HIST = 257;
struct Choice {
  unsigned T;
  int want;                  // of those equal to T, -1: all
};
template <class Keys>
__device__ Choice choose_threshold(int budget, int (&hist)[COPIES * HIST], int* sm, Keys each) {
  const int tid = threadIdx.x, lane = tid & 63, copy = (tid & (COPIES - 1)) * HIST;
  unsigned T = 0, mask = 0;
  int want = budget;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    for (int i = tid; i < COPIES * HIST; i += EV_THREADS) hist[i] = 0;
    __syncthreads();
    each([&](unsigned key) { if ((key & mask) == T) atomicAdd(&hist[copy + (key >> shift & 255)], 1); });
    __syncthreads();
    if (tid < 256) {
      int n = 0;
#pragma unroll
      for (int x = 0; x < COPIES; ++x) n += hist[x * HIST + tid];
      hist[tid] = n;         // (of this thread's own column)
    }
    __syncthreads();
    if (tid < 64) {                                     // from the top
      const int d0 = 255 - 4 * tid;
      int n[4], all = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) all += n[x] = hist[d0 - x];
      int sum = all;
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) {
        const int y = __shfl_up(sum, x, 64);
        if (lane >= x) sum += y;
      }
      int above = sum - all;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (above < want && above + n[x] >= want) {
          sm[0] = d0 - x;
          sm[1] = want - above;
          sm[2] = n[x];
        }
        above += n[x];
      }
    }
    __syncthreads();
    T |= (unsigned)sm[0] << shift;
    want = sm[1];
    mask |= 255u << shift;
    if (want == sm[2]) return {T, -1};
  }
  return {T, want};
}

// Up to EV_THREADS * KPT slots: the keys stay in registers, thread t has slots t, t + EV_THREADS, ..  Returns the number of moves.
template <int KPT>
__device__ int choose_in_registers(const Evict& e, Unit& u, int (&hist)[COPIES * HIST], int* sm) {
  int (*counts)[EV_WAVES] = reinterpret_cast<int (*)[EV_WAVES]>(hist);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, budget = e.budget;
  unsigned key[KPT];
  {
    float w[KPT];
    int pos[KPT], last = -2147483647 - 1;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int s = i * EV_THREADS + tid;
      w[i] = 0.f;
      pos[i] = -2147483647 - 1;
      if (s < u.len) {
        w[i] = u.w[s];
        pos[i] = u.pos[s];
      }
    }
#pragma unroll
    for (int i = 0; i < KPT; ++i) last = max(last, pos[i]);
    u.recent = (long long)largest_of_all(last, sm) - e.n_recent;
#pragma unroll
    for (int i = 0; i < KPT; ++i) key[i] = i * EV_THREADS + tid < u.len ? key_of(e, u, w[i], pos[i]) : 0u;     // (below every key there is)
  }
  const Choice choice = choose_threshold(budget, hist, sm, [&](auto add) {
#pragma unroll
    for (int i = 0; i < KPT; ++i)
      if (i * EV_THREADS + tid < u.len) add(key[i]);
  });
  const unsigned T = choice.T;
  const bool exact = choice.want < 0;
  const int want = choice.want;
  unsigned kept = 0;
  if (exact) {
#pragma unroll
    for (int i = 0; i < KPT; ++i) kept |= (unsigned)(key[i] >= T && i * EV_THREADS + tid < u.len) << i;
  } else {
    auto tie = [&](int i) { return key[i] == T && i * EV_THREADS + tid < u.len; };
    __syncthreads();
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const unsigned long long mask = __ballot(tie(i));
      if (lane == 0) counts[i][wave] = __popcll(mask);
    }
    __syncthreads();
    int rank = 0;                                                  // ties before these
#pragma unroll
    for (int i0 = 0; i0 < KPT; i0 += 4) {                          // sixteen lanes, one for each wave, to 1024 slots
      const int mine = counts[i0 + (lane >> 4)][lane & 15], sum = row_scan16(mine);
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int i = i0 + x, first = rank + __builtin_amdgcn_readlane(sum - mine, 16 * x + wave);
        rank += __builtin_amdgcn_readlane(sum, 16 * x + 15);
        const unsigned long long mask = __ballot(tie(i));
        kept |= (unsigned)((key[i] > T && i * EV_THREADS + tid < u.len) || (tie(i) && first + below(mask) < want)) << i;
      }
    }
  }
  // freed slots before the budget and kept ones behind it, numbered in slot order: 16 bits each (no more than half of the slots)
  auto moves = [&](int i) { return i * EV_THREADS + tid < u.len && (kept >> i & 1) != (unsigned)(i * EV_THREADS + tid < budget); };
  __syncthreads();
#pragma unroll
  for (int i = 0; i < KPT; ++i) {
    const unsigned long long all = __ballot(moves(i)), holes = __ballot(moves(i) && i * EV_THREADS + tid < budget);
    if (lane == 0) counts[i][wave] = __popcll(holes) | __popcll(all & ~holes) << 16;
  }
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int i0 = 0; i0 < KPT; i0 += 4) {
    const int mine = counts[i0 + (lane >> 4)][lane & 15], sum = row_scan16(mine);
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int i = i0 + x, s = i * EV_THREADS + tid, first = before + __builtin_amdgcn_readlane(sum - mine, 16 * x + wave);
      before += __builtin_amdgcn_readlane(sum, 16 * x + 15);
      const unsigned long long all = __ballot(moves(i)), holes = __ballot(moves(i) && s < budget);
      if (moves(i)) {
        if (s < budget) u.moves[(first & 0xffff) + below(holes)].y = s;
        else u.moves[(first >> 16) + below(all & ~holes)].x = s;
      }
    }
  }
  return before >> 16;
}

// Any number of slots: keys are formed anew in each pass.
__device__ int choose_in_passes(const Evict& e, Unit& u, int (&hist)[COPIES * HIST], int* sm) {
  const int tid = threadIdx.x, budget = e.budget;
  int last = -2147483647 - 1;
  for (int i = tid; i < u.len; i += EV_THREADS) last = max(last, u.pos[i]);
  u.recent = (long long)largest_of_all(last, sm) - e.n_recent;
  auto key_at = [&](int i) { return key_of(e, u, u.w[i], u.pos[i]); };
  const Choice choice = choose_threshold(budget, hist, sm, [&](auto add) {
    for (int i = tid; i < u.len; i += EV_THREADS) add(key_at(i));
  });
  const unsigned T = choice.T;
  const int want = choice.want < 0 ? 0 : choice.want;
  const bool exact = choice.want < 0;

  // in slot order: what is kept; the freed slots before the budget, then the kept ones behind it, paired as they come
  int ties = 0, holes = 0, movers = 0;
  for (int i0 = 0; i0 < u.len; i0 += EV_THREADS) {
    const int i = i0 + tid;
    const unsigned key = i < u.len ? key_at(i) : 0u;
    const bool tie = i < u.len && key == T;
    int total;
    const unsigned long long tie_mask = __ballot(tie);
    const int rank = ties + before_me(__popcll(tie_mask), sm, total) + below(tie_mask);
    ties += total;
    const bool kept = i < u.len && (exact ? key >= T : key > T || (tie && rank < want));
    const bool hole = i < budget && !kept, mover = i >= budget && kept;
    const unsigned long long hole_mask = __ballot(hole), mover_mask = __ballot(mover);
    const int at = before_me(__popcll(hole_mask) | __popcll(mover_mask) << 16, sm, total);
    if (hole) u.moves[holes + (at & 0xffff) + below(hole_mask)].y = i;
    if (mover) u.moves[movers + (at >> 16) + below(mover_mask)].x = i;
    holes += total & 0xffff;
    movers += total >> 16;
  }
  return movers;
}

__global__ __launch_bounds__(EV_THREADS) void choose_kernel(Evict e) {
  __shared__ int hist[COPIES * HIST], sm[EV_WAVES];
  const Pages& p = e.p;
  const int unit = blockIdx.x, b = unit / p.Hkv, h = unit % p.Hkv, tid = threadIdx.x;
  const int len = p.lens[b], budget = e.budget;
  bool ok = len >= 0 && len <= p.cap;
  if (ok && len > budget) {
    const int32_t* table = p.table + (size_t)b * p.width;
    bool bad = false;
    for (int i = tid; i < (len + (1 << p.bits) - 1) >> p.bits; i += EV_THREADS) bad |= table[i] < 0 || table[i] >= p.pages;
    ok = !__syncthreads_or(bad);
  }
  if (h == 0 && tid == 0 && e.status) e.status[b] = ok ? TREEKV_OK : TREEKV_EINVAL;
  if (!ok || len <= budget) {
    if (tid == 0) e.count[unit] = -1;
    return;
  }
  Unit u = {p.weights + track_row(p, b, h), p.positions + track_row(p, b, h), e.moves + (size_t)unit * e.stride, len, 0};
  int count;
  // (8 x 32 units of 4097 slots: 13.9 us with 8 keys a thread, 22.6 with 32; of 10000 45 with 32)
  if (len <= 4 * EV_THREADS) count = choose_in_registers<4>(e, u, hist, sm);
  else if (len <= 8 * EV_THREADS) count = choose_in_registers<8>(e, u, hist, sm);
  else if (len <= 32 * EV_THREADS) count = choose_in_registers<32>(e, u, hist, sm);
  else count = choose_in_passes(e, u, hist, sm);
  if (tid == 0) e.count[unit] = count;
}

// 2^piece_bits lanes copy a token: keys, values, weight and position.  grid: `parts` workgroups per unit.
__global__ __launch_bounds__(MV_THREADS) void move_kernel(Evict e, int parts, int piece_bits) {
  const Pages& p = e.p;
  const int unit = (int)(blockIdx.x / parts), part = (int)(blockIdx.x % parts), b = unit / p.Hkv, h = unit % p.Hkv;
  const int count = e.count[unit], tid = threadIdx.x;
  if (part == 0 && h == 0 && tid == 0) e.lens_out[b] = count < 0 ? p.lens[b] : e.budget;
  if (count < 0) return;
  const int piece = tid & ((1 << piece_bits) - 1), step = MV_THREADS >> piece_bits;
  const int32_t* table = p.table + (size_t)b * p.width;
  const int2* moves = e.moves + (size_t)unit * e.stride;
  const size_t track = track_row(p, b, h);
  for (int i = part * step + (tid >> piece_bits); i < count; i += parts * step) {
    const int2 m = moves[i];
    const size_t from = ((pool_row(p, table[m.x >> p.bits], h, m.x) << piece_bits) + piece) << 4;
    const size_t to = ((pool_row(p, table[m.y >> p.bits], h, m.y) << piece_bits) + piece) << 4;
    const uint4 k = *reinterpret_cast<const uint4*>(p.k + from), v = *reinterpret_cast<const uint4*>(p.v + from);
    *reinterpret_cast<uint4*>(p.k + to) = k;
    *reinterpret_cast<uint4*>(p.v + to) = v;
    if (piece == 0) {
      p.weights[track + m.y] = p.weights[track + m.x];
      p.positions[track + m.y] = p.positions[track + m.x];
    }
  }
}

}  // namespace

size_t paged_evict_scratch_bytes(const treekv_paged_cache& c) {
  const size_t units = (size_t)c.batch * c.kv_heads, most = (size_t)c.table_width * c.page_size / 2;
  return align_up(units * 4) + align_up(units * most * sizeof(int2));
}

int launch_paged_evict(const treekv_paged_cache& c, int budget, int n_sink, int n_recent, int32_t* lens_out, void* scratch, int32_t* status,
                       hipStream_t s) {
  const size_t units = (size_t)c.batch * c.kv_heads;
  Evict e;
  e.p = pages_of(c);
  e.budget = budget; e.n_sink = n_sink; e.n_recent = n_recent;
  e.count = (int*)scratch;
  e.moves = (int2*)((char*)scratch + align_up(units * 4));
  e.status = status;
  e.lens_out = lens_out ? lens_out : c.lens;
  e.stride = budget >= e.p.cap ? 0 : budget < e.p.cap - budget ? budget : e.p.cap - budget;
  hipLaunchKernelGGL(choose_kernel, dim3((unsigned)units), dim3(EV_THREADS), 0, s, e);
  const int piece_bits = __builtin_ctz(c.head_dim * (c.dtype == TREEKV_F32 ? 4 : 2) / 16);
  // most moves a unit can have, MV_THREADS >> piece_bits at a time, and about eight workgroups a compute unit over all units
  const int step = MV_THREADS >> piece_bits;
  const long long fill = (2048 + (long long)units - 1) / (long long)units, need = e.stride > 0 ? (e.stride + step - 1) / step : 1;
  const int parts = (int)(need < fill ? need : fill);
  hipLaunchKernelGGL(move_kernel, dim3((unsigned)(units * parts)), dim3(MV_THREADS), 0, s, e, parts, piece_bits);
  return finish_launch();
}

}  // namespace tkv
