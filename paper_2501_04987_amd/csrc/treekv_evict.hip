// Eviction from a paged cache by accumulated weight (treekv_paged_evict) for gfx950.
//
// A unit is one KV head of one sequence.  Of its len tokens the `budget` first by (protected, weight descending, slot) are kept:
//   key     an order-preserving 32-bit image of the weight; protected tokens above all, NaNs as minus infinity
//   choice  the budget-th largest key T by four rounds of 8 bits (a histogram in LDS each), then, in slot order, whatever is
//           above T and the first of what equals it
//   move    attention does not ask for the order of columns, so what is kept stays where it is: only tokens from slots behind
//           the budget move, into the freed slots before it, as many rows as were kept there (of a decode step one, where
//           closing the gaps would move half of the cache)
// Two kernels: one workgroup per unit makes the choice and lists the moves, then all of the chip copies the rows.

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
  int32_t* status;
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

__global__ __launch_bounds__(EV_THREADS) void choose_kernel(Evict e) {
  __shared__ int hist[256], sm[EV_WAVES], found[2];
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
  const float* w = p.weights + track_row(p, b, h);
  const int32_t* pos = p.positions + track_row(p, b, h);
  int last = -2147483647 - 1;
  for (int i = tid; i < len; i += EV_THREADS) last = max(last, pos[i]);
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) last = max(last, __shfl_xor(last, x, 64));
  if ((tid & 63) == 0) sm[tid >> 6] = last;
  __syncthreads();
  for (int i = 0; i < EV_WAVES; ++i) last = max(last, sm[i]);
  const long long recent = (long long)last - e.n_recent;
  auto key_of = [&](int i) { return pos[i] < e.n_sink || pos[i] > recent ? 0xffffffffu : order_of(w[i]); };

  // T and how many of those equal to it are kept
  unsigned T = 0, mask = 0;
  int want = budget;
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (tid < 256) hist[tid] = 0;
    __syncthreads();
    for (int i = tid; i < len; i += EV_THREADS) {
      const unsigned key = key_of(i);
      if ((key & mask) == T) atomicAdd(&hist[key >> shift & 255], 1);
    }
    __syncthreads();
    if (tid < 64) {                                     // from the top: the digit where `want` is reached
      const int d0 = 255 - 4 * tid;
      int n[4], all = 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) all += n[x] = hist[d0 - x];
      int sum = all;
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) {
        const int y = __shfl_up(sum, x, 64);
        if (tid >= x) sum += y;
      }
      int above = sum - all;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        if (above < want && above + n[x] >= want) {
          found[0] = d0 - x;
          found[1] = want - above;
        }
        above += n[x];
      }
    }
    __syncthreads();
    T |= (unsigned)found[0] << shift;
    want = found[1];
    mask |= 255u << shift;
  }

  // in slot order: what is kept; the freed slots before the budget, then the kept ones behind it, paired as they come
  int2* moves = e.moves + (size_t)unit * e.stride;
  int ties = 0, holes = 0, movers = 0;
  for (int i0 = 0; i0 < len; i0 += EV_THREADS) {
    const int i = i0 + tid;
    const unsigned key = i < len ? key_of(i) : 0u;
    const bool tie = i < len && key == T;
    int total;
    const unsigned long long tie_mask = __ballot(tie);
    const int rank = ties + before_me(__popcll(tie_mask), sm, total) + below(tie_mask);
    ties += total;
    const bool kept = i < len && (key > T || (tie && rank < want));
    const bool hole = i < budget && !kept, mover = i >= budget && kept;
    const unsigned long long hole_mask = __ballot(hole), mover_mask = __ballot(mover);
    const int at = before_me(__popcll(hole_mask) | __popcll(mover_mask) << 16, sm, total);
    if (hole) moves[holes + (at & 0xffff) + below(hole_mask)].y = i;
    if (mover) moves[movers + (at >> 16) + below(mover_mask)].x = i;
    holes += total & 0xffff;
    movers += total >> 16;
  }
  if (tid == 0) e.count[unit] = movers;
}

// 2^piece_bits lanes copy a token: keys, values, weight and position.  grid: `parts` workgroups per unit.
__global__ __launch_bounds__(MV_THREADS) void move_kernel(Evict e, int parts, int piece_bits) {
  const Pages& p = e.p;
  const int unit = (int)(blockIdx.x / parts), part = (int)(blockIdx.x % parts), b = unit / p.Hkv, h = unit % p.Hkv;
  const int count = e.count[unit], tid = threadIdx.x;
  if (count < 0) return;
  if (part == 0 && h == 0 && tid == 0) p.lens[b] = e.budget;
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

int launch_paged_evict(const treekv_paged_cache& c, int budget, int n_sink, int n_recent, void* scratch, int32_t* status, hipStream_t s) {
  const size_t units = (size_t)c.batch * c.kv_heads;
  Evict e;
  e.p = pages_of(c);
  e.budget = budget; e.n_sink = n_sink; e.n_recent = n_recent;
  e.count = (int*)scratch;
  e.moves = (int2*)((char*)scratch + align_up(units * 4));
  e.status = status;
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
