// treekv_fork: sequences of one context become copies of sequences of another, on the device and without scratch.
//
// A unit's state is its cache rows, scores, order arrays and bookkeeping words, each copied as it lies: slots keep their
// numbers, so that the copy goes on bit for bit as its source would.  A cache that is still filling has its n tokens in
// slots 0 .. n-1; the rows behind them, and all rows of a sequence that is emptied, become zeros, as a reset leaves them: the
// decode and chunk kernels multiply rows behind the last one by probabilities of zero, and what the sequence before left there
// may be an infinity or a NaN.  Bound by memory: every live byte once in, every row once out (one sequence
// of 8 heads x 4096 rows x 128 into 15: 65 us, 252 MB written at 3.9 TB/s; stored past the caches 62, but the read of the
// copies that follows takes 11 longer).  The zeros are: 12 sequences of that size emptied beside one copied and the whole
// exported 92 us, 128 through the caches.

#include "treekv_internal.h"

namespace tkv {

namespace {

constexpr int FORK_THREADS = 256;
constexpr int FORK_VECS = 4;                       // 16-byte pieces of K, and of V, a thread copies
constexpr int FORK_PAIRS = 64;                     // per launch: they travel as kernel arguments

struct ForkPairs {
  int src[FORK_PAIRS], dst[FORK_PAIRS];
};

// grid (pieces + 1, pairs * Hkv): the workgroups with blockIdx.x = 0 take the order arrays, scores and bookkeeping words.
__global__ __launch_bounds__(FORK_THREADS) void fork_kernel(Params to, Params from, ForkPairs pairs, int row_vec) {
  const int pair = blockIdx.y / to.Hkv, head = blockIdx.y % to.Hkv, tid = threadIdx.x;
  const int s = pairs.src[pair], d = pairs.dst[pair];
  if (to.K == from.K && s == d) return;
  const size_t du = (size_t)d * to.Hkv + head, su = (size_t)(s < 0 ? 0 : s) * to.Hkv + head;
  const int* meta = from.meta + su * META_STRIDE;
  const int m = to.m, r = max(to.n_recent, 1), cap = to.cap;
  if (blockIdx.x == 0) {
    int* Ed = to.E + du * 2 * m;
    int* PEd = to.PE + du * 2 * m;
    int* Rd = to.R + du * r;
    float* Sd = to.S + du * cap;
    int* meta_d = to.meta + du * META_STRIDE;
    if (s < 0) {                                   // as after a reset
      for (int i = tid; i < 2 * m; i += FORK_THREADS) Ed[i] = PEd[i] = i < m ? to.n_sink + i : 0;
      for (int i = tid; i < to.n_recent; i += FORK_THREADS) Rd[i] = to.n_sink + m + i;
      for (int i = tid; i < cap; i += FORK_THREADS) Sd[i] = 0.f;
      if (tid < META_STRIDE) meta_d[tid] = 0;
      return;
    }
    const int* Es = from.E + su * 2 * m;
    const int* PEs = from.PE + su * 2 * m;
    const int* Rs = from.R + su * r;
    const float* Ss = from.S + su * cap;
    for (int i = tid; i < 2 * m; i += FORK_THREADS) { Ed[i] = Es[i]; PEd[i] = PEs[i]; }
    for (int i = tid; i < to.n_recent; i += FORK_THREADS) Rd[i] = Rs[i];
    for (int i = tid; i < cap; i += FORK_THREADS) Sd[i] = Ss[i];
    if (tid < META_STRIDE) meta_d[tid] = meta[tid];
    return;
  }
  const int n = s < 0 ? 0 : meta[META_N];
  const size_t vecs = (size_t)(n < to.budget ? n : cap) * row_vec, all = (size_t)cap * row_vec;
  const uint4* Ks = reinterpret_cast<const uint4*>(from.K) + su * cap * row_vec;
  const uint4* Vs = reinterpret_cast<const uint4*>(from.V) + su * cap * row_vec;
  uint4* Kd = reinterpret_cast<uint4*>(to.K) + du * cap * row_vec;
  uint4* Vd = reinterpret_cast<uint4*>(to.V) + du * cap * row_vec;
  const size_t base = (size_t)(blockIdx.x - 1) * FORK_THREADS * FORK_VECS + tid;
#pragma unroll
  for (int x = 0; x < FORK_VECS; ++x) {
    const size_t i = base + (size_t)x * FORK_THREADS;
    if (i < vecs) { Kd[i] = Ks[i]; Vd[i] = Vs[i]; }
    else if (i < all) {                            // past the caches, where they would only be in the way
      store16<true>(Kd + i, make_uint4(0, 0, 0, 0));
      store16<true>(Vd + i, make_uint4(0, 0, 0, 0));
    }
  }
}

}  // namespace

int launch_fork(const Params& to, const Params& from, const int32_t* src, const int32_t* dst, int count, hipStream_t s) {
  const int row_vec = to.D * (to.dtype == TREEKV_BF16 ? 2 : 4) / 16;
  const size_t pieces = ((size_t)to.cap * row_vec + FORK_THREADS * FORK_VECS - 1) / (FORK_THREADS * FORK_VECS);
  for (int i0 = 0; i0 < count; i0 += FORK_PAIRS) {
    const int n = count - i0 < FORK_PAIRS ? count - i0 : FORK_PAIRS;
    ForkPairs pairs;
    for (int i = 0; i < FORK_PAIRS; ++i) {
      pairs.src[i] = i < n ? src[i0 + i] : -1;
      pairs.dst[i] = i < n ? dst[i0 + i] : 0;
    }
    hipLaunchKernelGGL(fork_kernel, dim3((unsigned)pieces + 1, n * to.Hkv), dim3(FORK_THREADS), 0, s, to, from, pairs, row_vec);
  }
  return finish_launch();
}

}  // namespace tkv
