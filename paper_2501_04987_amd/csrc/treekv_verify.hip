// treekv_tree_verify: the accepted path of a drafted tree and the token that follows it, for gfx950.
//
// The nodes come after their parents, so one walk over them in order meets the children of the last accepted token, and after
// an acceptance the new one's.  With P the target's row there and Q the drafter's, k refusals leave
//   P_k = max(P - c_k Q, 0) / W_k,   W_k = sum of max(P - c_k Q, 0),   c_1 = 1,  c_k+1 = c_k + W_k
// (each step subtracts Q from what the last one made sum to 1, that is, W_k times Q from what it was made of), so a refusal is
// one pass over two rows, whatever came before it, and the next child is accepted if u Q(x) W_k < max(P(x) - c_k Q(x), 0).
// Sums are in double, 2^14 terms a lane at most: off by 2^-39 of themselves, 2^-15 of half a step of fp32.  A difference is off by
// 2^-53 of c_k Q, so k refusals leave P_k good to k 2^-52 (terms of W_k) / W_k or better: W_k is the part of the first P that they
// leave, and an error of c_k does not grow, for W_k falls where c_k rises.  (The rule step by step multiplies its roundings by what
// each refusal takes.)
//
// Bound by latency: 16 trees of 26 nodes over 131072 tokens 29-43 us (the rows take 3 at the rate of memory), four kernels that each
// wait for the state, its sums and the rows; a chain of 5 over 32000 tokens 12-14 us.
//
// A sequence's rows are split among waves; the token that follows is found by the waves' sums, then among parts of the one it
// lies in, then by a scan.

#include "treekv_internal.h"

namespace tkv {

namespace {

constexpr int VF_THREADS = 1024, VF_WAVES = VF_THREADS / 64;

__device__ inline double positive(float x) { return x > 0.f ? (double)x : 0.0; }
__device__ inline float value_at(const uint16_t* row, int x) { return __uint_as_float((unsigned)row[x] << 16); }
__device__ inline float value_at(const float* row, int x) { return row[x]; }

// What is left of a row: P - c Q above 0, without the tokens that were taken out.
template <typename T>
struct Left {
  static constexpr int EPL = Storage<T>::EPL;
  const T *p, *q;                   // q: null if nothing of it is subtracted
  double c;
  int vocab, skew;                  // elements by which the rows begin behind a 16-byte boundary
  const int* out;                   // tokens taken out
  int n_out;
  __device__ int pieces() const { return (vocab + skew + EPL - 1) / EPL; }
  struct Piece {
    float a[EPL], b[EPL];
  };
  // Pieces [first_whole(), whole_end()) lie in the rows from end to end.
  __device__ int first_whole() const { return skew ? 1 : 0; }
  __device__ int whole_end() const { return (vocab + skew) / EPL; }
  template <bool SUB>
  __device__ Piece load_whole(int j) const {
    Piece u;
    Storage<T>::widen(*reinterpret_cast<const uint4*>(p + (j * EPL - skew)), u.a);
    if constexpr (SUB) Storage<T>::widen(*reinterpret_cast<const uint4*>(q + (j * EPL - skew)), u.b);
    return u;
  }
  // Any piece; what is no part of the rows is 0.
  __device__ Piece load(int j) const {
    if (j >= first_whole() && j < whole_end()) return q ? load_whole<true>(j) : load_whole<false>(j);
    Piece u;
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      const int x = j * EPL - skew + e;
      u.a[e] = x >= 0 && x < vocab ? value_at(p, x) : 0.f;
      u.b[e] = x >= 0 && x < vocab && q ? value_at(q, x) : 0.f;
    }
    return u;
  }
  __device__ void values(int j, const Piece& u, double (&y)[EPL]) const {
#pragma unroll
    for (int e = 0; e < EPL; ++e) y[e] = q ? fmax(positive(u.a[e]) - c * positive(u.b[e]), 0.0) : positive(u.a[e]);
    for (int i = 0; i < n_out; ++i) {
      const int e0 = out[i] - (j * EPL - skew);
      if (e0 >= 0 && e0 < EPL)
#pragma unroll
        for (int e = 0; e < EPL; ++e)
          if (e == e0) y[e] = 0.0;
    }
  }
  __device__ void piece(int j, double (&y)[EPL]) const { values(j, load(j), y); }
};

__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) v += __shfl_xor(v, x, 64);
  return v;
}
template <typename T, bool SUB>
__device__ inline double sum_whole(const Left<T>& l, int lo, int hi) {
  constexpr int AHEAD = 4, EPL = Left<T>::EPL;         // pieces a lane has on their way at once
  double sum = 0.0;
  for (int j0 = lo + (int)(threadIdx.x & 63); j0 < hi; j0 += 64 * AHEAD) {
    typename Left<T>::Piece u[AHEAD];
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) u[x] = l.template load_whole<SUB>(min(j0 + 64 * x, hi - 1));
#pragma unroll
    for (int x = 0; x < AHEAD; ++x) {
      double y[EPL], mine = 0.0;
      l.values(min(j0 + 64 * x, hi - 1), u[x], y);
#pragma unroll
      for (int e = 0; e < EPL; ++e) mine += y[e];
      sum += j0 + 64 * x < hi ? mine : 0.0;
    }
  }
  return sum;
}
// Pieces [lo, hi) summed by the wave.
template <typename T>
__device__ inline double sum_pieces(const Left<T>& l, int lo, int hi) {
  const int first = max(lo, l.first_whole()), end = min(hi, l.whole_end());
  double sum = l.q ? sum_whole<T, true>(l, first, end) : sum_whole<T, false>(l, first, end);
  // a piece at either end of the rows that is cut (one of a short row is both)
  const int lane = threadIdx.x & 63, cut = lane == 0 ? 0 : l.pieces() - 1;
  if (lane < (l.pieces() > 1 ? 2 : 1) && cut >= lo && cut < hi && (cut < first || cut >= end)) {
    double y[Left<T>::EPL];
    l.piece(cut, y);
#pragma unroll
    for (int e = 0; e < Left<T>::EPL; ++e) sum += y[e];
  }
  return wave_sum(sum);
}
__device__ inline int part_at(int lo, int hi, int part, int parts) { return lo + (int)((long long)(hi - lo) * part / parts); }

// Sums of the VF_WAVES parts of pieces [lo, hi) into sm; all threads get the total.
template <typename T>
__device__ inline double sum_parts(const Left<T>& l, int lo, int hi, double* sm) {
  const int wave = threadIdx.x >> 6;
  const double s = sum_pieces(l, part_at(lo, hi, wave, VF_WAVES), part_at(lo, hi, wave + 1, VF_WAVES));
  __syncthreads();
  if ((threadIdx.x & 63) == 0) sm[wave] = s;
  __syncthreads();
  double total = 0.0;
  for (int i = 0; i < VF_WAVES; ++i) total += sm[i];
  return total;
}
// The part in which the sum passes t, `before` what comes before it; the last that is not empty if it does not.
__device__ inline int choose_part(const double* sm, double t, double& before) {
  int last = -1;
  double sum = before, at = before;
  for (int i = 0; i < VF_WAVES; ++i) {
    if (sm[i] > 0.0) {
      last = i;
      at = sum;
      if (sum + sm[i] > t) break;
    }
    sum += sm[i];
  }
  before = at;
  return last;
}

// The smallest token with something left whose sum passes u * total, by all threads; sm holds the sums of the parts.
template <typename T>
__device__ inline int draw(const Left<T>& l, double u, double total, double* sm, int* found) {
  const double t = u * total;
  double before = 0.0;
  int lo = 0, hi = l.pieces(), part = choose_part(sm, t, before);
  if (part < 0) return -1;
  const int lo1 = part_at(lo, hi, part, VF_WAVES), hi1 = part_at(lo, hi, part + 1, VF_WAVES);
  sum_parts(l, lo1, hi1, sm);
  part = choose_part(sm, t, before);
  if (part < 0) return -1;
  const int lane = threadIdx.x & 63;
  if (threadIdx.x < 64) {
    int last = -1;
    const int end = part_at(lo1, hi1, part + 1, VF_WAVES);
    for (int j0 = part_at(lo1, hi1, part, VF_WAVES); j0 < end; j0 += 64) {
      double y[Left<T>::EPL], mine = 0.0;
      int tail = -1;
      if (j0 + lane < end) {
        l.piece(j0 + lane, y);
#pragma unroll
        for (int e = 0; e < Left<T>::EPL; ++e) {
          mine += y[e];
          if (y[e] > 0.0) tail = (j0 + lane) * Left<T>::EPL - l.skew + e;
        }
      }
      double sum = mine;
#pragma unroll
      for (int x = 1; x < 64; x <<= 1) {
        const double z = __shfl_up(sum, x, 64);
        if (lane >= x) sum += z;
      }
      const unsigned long long hit = __ballot(mine > 0.0 && before + sum > t), any = __ballot(mine > 0.0);
      if (hit) {
        const int first = __ffsll((long long)hit) - 1;
        double at = before + (sum - mine);
        int x = -1;
        if (lane == first) {
#pragma unroll
          for (int e = 0; e < Left<T>::EPL; ++e) {
            at += y[e];
            if (x < 0 && y[e] > 0.0 && at > t) x = (j0 + lane) * Left<T>::EPL - l.skew + e;
          }
          if (x < 0) x = tail;
        }
        last = __shfl(x, first, 64);
        break;
      }
      if (any) last = __shfl(tail, 63 - __clzll((long long)any), 64);
      before += __shfl(sum, 63, 64);
    }
    if (lane == 0) *found = last;
  }
  __syncthreads();
  return *found;
}

// What the walk has come to.  Between kernels it lies in scratch (the tokens taken out behind it).
struct State {
  double c, W, next_c;               // of P_k; next_c: of the pass that is asked for
  int at, len, i;                    // last accepted node, accepted ones, next node
  int asked;                         // 0: nothing; 1: W for next_c, after a refusal; 2: the sums of what is left; 3: all is done
  int subtracted, n_out;
  int sums;                          // which of the two sets of partial sums is what is left's
};

// A sequence's tree.  What the distributions after a node's parent say of its token is known before the walk, so all of them are read
// at once and the walk waits for none.
struct Nodes {
  int parent[TREEKV_TREE_MAX_NODES];                   // -2 also where the token is none
  int token[TREEKV_TREE_MAX_NODES], out[TREEKV_TREE_MAX_NODES];
  float p[TREEKV_TREE_MAX_NODES], q[TREEKV_TREE_MAX_NODES], uniform[TREEKV_TREE_MAX_NODES + 1];
};
template <typename T>
__device__ inline void load_nodes(Nodes& sm, const treekv_verify_args& a, int b) {
  for (int i = threadIdx.x; i < a.n; i += blockDim.x) {
    int parent = a.parents[(size_t)b * a.n + i];
    const int x = a.tokens[(size_t)b * a.n + i];
    if (parent < -1 || parent >= i || x < 0 || x >= a.vocab) parent = -2;
    sm.parent[i] = parent;
    sm.token[i] = x;
    if (parent != -2) {
      const size_t at = ((size_t)b * (a.n + 1) + parent + 1) * a.vocab + x;
      sm.p[i] = value_at((const T*)a.target + at, 0);
      if (a.draft) sm.q[i] = value_at((const T*)a.draft + at, 0);
    }
  }
  for (int i = threadIdx.x; i <= a.n; i += blockDim.x) sm.uniform[i] = a.uniforms[(size_t)b * (a.n + 1) + i];
}

template <typename T>
struct Walk {
  const treekv_verify_args& a;
  State& s;
  const int b;
  Nodes& nodes;                      // of the sequence, in LDS
  bool writes;                       // this thread writes the path
  int parent[TREEKV_TREE_MAX_NODES / 64];              // of nodes lane, lane + 64, ..
  Left<T> l;
  const T* draft;

  __device__ void rows() {           // of the last accepted node, less what has been subtracted
    const size_t row = ((size_t)b * (a.n + 1) + s.at + 1) * a.vocab;
    l.p = (const T*)a.target + row;
    draft = a.draft ? (const T*)a.draft + row : nullptr;
    l.q = s.subtracted ? draft : nullptr;
    l.c = s.c;
    l.vocab = a.vocab;
    l.skew = (int)(row % Left<T>::EPL);
    l.out = nodes.out;
    l.n_out = s.n_out;
  }
  __device__ void enter(int node) {
    s.at = node;
    s.c = 0.0;
    s.W = 1.0;
    s.subtracted = s.n_out = 0;
    rows();
  }
  // What a pass is asked about.
  __device__ Left<T> asked() const {
    Left<T> x = l;
    if (s.asked == 1) {
      x.q = draft;
      x.c = s.next_c;
    }
    return x;
  }
  // The pass's sum.  Returns whether it is that of what is left now.
  __device__ bool answer(double sum) {
    const bool refused = s.asked == 1;
    s.asked = 0;
    if (refused) {
      if (!(sum > 0.0)) return false;                  // P stays
      s.c = s.next_c;
      s.subtracted = 1;
      rows();
    }
    s.W = sum;
    return true;
  }
  __device__ void look() {
#pragma unroll
    for (int x = 0; x < TREEKV_TREE_MAX_NODES / 64; ++x) {
      const int i = 64 * x + (int)(threadIdx.x & 63);
      parent[x] = i < a.n ? nodes.parent[i] : -2;
    }
  }
  // The first child of the last accepted token from node i on; n if there is none.
  __device__ int child(int i) const {
    int found = a.n;
#pragma unroll
    for (int x = TREEKV_TREE_MAX_NODES / 64 - 1; x >= 0; --x) {
      const unsigned long long from = i <= 64 * x ? ~0ull : i >= 64 * x + 64 ? 0ull : ~0ull << (i - 64 * x);
      const unsigned long long hit = __ballot(parent[x] == s.at) & from;
      if (hit) found = 64 * x + __ffsll((long long)hit) - 1;
    }
    return found;
  }
  // On to the next refusal that asks for a pass, or to the end.  All threads of the workgroup; returns false at the end.
  __device__ bool on() {
    for (; (s.i = child(s.i)) < a.n; ++s.i) {
      const int x = nodes.token[s.i];
      const double u = nodes.uniform[s.i], p = positive(nodes.p[s.i]);
      bool accepted;
      if (draft) {
        const double q = positive(nodes.q[s.i]);
        accepted = u * q * s.W < fmax(p - s.c * q, 0.0);
      } else {
        bool gone = false;
        for (int j = 0; j < s.n_out; ++j) gone |= nodes.out[j] == x;
        accepted = u * s.W < (gone ? 0.0 : p);
        if (!accepted && !gone) {
          s.W = fmax(s.W - p, 0.0);
          __syncthreads();
          if (threadIdx.x == 0) nodes.out[s.n_out] = x;
          __syncthreads();
          l.n_out = ++s.n_out;
        }
      }
      if (accepted) {
        if (writes) a.path[(size_t)b * a.n + s.len] = s.i;
        ++s.len;
        enter(s.i);
      } else if (draft) {
        s.next_c = s.c + s.W;
        s.asked = 1;
        ++s.i;
        return true;
      }
    }
    return false;
  }
};

// Few sequences over many tokens: passes by VF_WAVES workgroups a sequence, one pass a kernel.  Each of them walks the same way and
// sums its part of the pass that comes out; the next kernel adds the parts.  After ROUNDS of these verify_kernel goes on by itself.
constexpr int PART_THREADS = 256, ROUNDS = 3;
struct Scratch {
  State* state;                      // [2][batch]
  int* out;                          // [2][batch][MAX_NODES]
  double* sums;                      // [2][batch][VF_WAVES]
};
inline size_t scratch_of(Scratch& x, char* at, int batch) {
  const size_t state = align_up((size_t)2 * batch * sizeof(State)), out = align_up((size_t)2 * batch * TREEKV_TREE_MAX_NODES * 4);
  x.state = (State*)at;
  x.out = (int*)(at + state);
  x.sums = (double*)(at + state + out);
  return state + out + align_up((size_t)2 * batch * VF_WAVES * 8);
}
// The state before round `round` and the answer to what it asked.
template <typename T>
__device__ inline void take_up(Walk<T>& w, const Scratch& x, int round, double (&sums)[VF_WAVES]) {
  const int set = round & 1, batch = w.a.batch;
  for (int i = 0; i < VF_WAVES; ++i) sums[i] = x.sums[((size_t)set * batch + w.b) * VF_WAVES + i];     // (read by then or not)
  w.s = x.state[set * batch + w.b];
  for (int i = threadIdx.x; i < w.s.n_out; i += blockDim.x) w.nodes.out[i] = x.out[((size_t)set * batch + w.b) * TREEKV_TREE_MAX_NODES + i];
  if (w.s.asked == 1 || w.s.asked == 2) {
    w.s.sums = set;
    double total = 0.0;
    for (int i = 0; i < VF_WAVES; ++i) total += sums[i];
    w.rows();
    if (w.answer(total)) {
      if (w.s.i >= w.a.n) w.s.asked = 3;
    } else {
      w.s.sums = -1;
    }
  } else {
    w.rows();
  }
  __syncthreads();
  w.look();
}

template <typename T>
__global__ __launch_bounds__(PART_THREADS) void verify_part_kernel(treekv_verify_args a, Scratch x, int round) {
  __shared__ Nodes sm;
  __shared__ double parts[PART_THREADS / 64];
  const int part = blockIdx.x % VF_WAVES, b = blockIdx.x / VF_WAVES, tid = threadIdx.x;
  load_nodes<T>(sm, a, b);
  State s = {};
  s.at = -1;
  s.W = 1.0;
  s.sums = -1;
  Walk<T> w = {a, s, b, sm, part == 0 && tid == 0, {}, {}, nullptr};
  double sums[VF_WAVES];
  if (round > 0) take_up(w, x, round, sums);
  else {
    w.enter(-1);
    __syncthreads();
    w.look();
  }
  if (s.asked != 3) {
    const bool fresh_sums = s.sums >= 0;               // the sums of what is left, if nothing more happens to it
    const int at = s.at, taken = s.n_out;
    if (!w.on()) s.asked = fresh_sums && s.at == at && s.n_out == taken ? 3 : 2;
    if (s.asked != 3) {
      const Left<T> l = w.asked();
      const int pieces = l.pieces(), lo = part_at(0, pieces, part, VF_WAVES), hi = part_at(0, pieces, part + 1, VF_WAVES), wave = tid >> 6;
      const double mine = sum_pieces(l, part_at(lo, hi, wave, PART_THREADS / 64), part_at(lo, hi, wave + 1, PART_THREADS / 64));
      if ((tid & 63) == 0) parts[wave] = mine;
      __syncthreads();
      if (tid == 0) {
        double sum = 0.0;
        for (int i = 0; i < PART_THREADS / 64; ++i) sum += parts[i];
        x.sums[((size_t)((round + 1) & 1) * a.batch + b) * VF_WAVES + part] = sum;
      }
    }
  }
  if (part == 0) {
    const size_t to = (size_t)((round + 1) & 1) * a.batch + b;
    for (int i = tid; i < s.n_out; i += PART_THREADS) x.out[to * TREEKV_TREE_MAX_NODES + i] = sm.out[i];
    if (tid == 0) x.state[to] = s;
  }
}

// A workgroup a sequence: the walk (or what is left of it after `rounds`), then the token that follows.
template <typename T>
__global__ __launch_bounds__(VF_THREADS) void verify_kernel(treekv_verify_args a, Scratch x, int rounds) {
  __shared__ Nodes sm;
  __shared__ double parts[VF_WAVES];
  __shared__ int found;
  const int b = blockIdx.x, tid = threadIdx.x;
  load_nodes<T>(sm, a, b);
  State s = {};
  s.at = -1;
  s.W = 1.0;
  s.sums = -1;
  Walk<T> w = {a, s, b, sm, tid == 0, {}, {}, nullptr};
  bool summed = false;               // `parts` holds the sums of what is left now
  if (rounds > 0) {
    double sums[VF_WAVES];
    take_up(w, x, rounds, sums);
    if (s.sums >= 0) {
      if (tid < VF_WAVES) parts[tid] = x.sums[((size_t)s.sums * a.batch + b) * VF_WAVES + tid];
      summed = true;
    }
    __syncthreads();
  } else {
    w.enter(-1);
    __syncthreads();
    w.look();
  }
  if (s.asked != 3)
    for (;;) {
      const int at = s.at, taken = s.n_out;
      const bool more = w.on();
      summed &= s.at == at && s.n_out == taken;
      if (!more) break;
      const Left<T> l = w.asked();
      summed = w.answer(sum_parts(l, 0, l.pieces(), parts));
    }
  double total = s.W;
  if (!summed) total = sum_parts(w.l, 0, w.l.pieces(), parts);
  if (!(total > 0.0) && (s.subtracted || s.n_out)) {
    w.enter(s.at);
    total = sum_parts(w.l, 0, w.l.pieces(), parts);
  }
  const int next = draw(w.l, (double)sm.uniform[a.n], total, parts, &found);
  for (int i = s.len + tid; i < a.n; i += VF_THREADS) a.path[(size_t)b * a.n + i] = -1;
  if (tid == 0) {
    a.path_len[b] = s.len;
    a.next_token[b] = next;
  }
}

// Rounds of parts where a sequence's own workgroup would read long rows while most of the chip idles.
// (16 trees of 26 nodes over 131072 tokens: 48.5 us without rounds, 29.5 with 3, 33 with 4, 38.5 with 6; a chain of 5 over 32000 12.1
// without, 20.4 with.)  Without the drafter's probabilities there is one pass.  About the border, without and with: 16 trees in
// bf16 over 50000 31.8 and 28.3, 65536 33.4 and 30.7, 98304 62 and 49; 64 trees 40.8 and 45.2, 34.4 and 37.0, 44.0 and 38.1;
// one 16.8 and 21.4, 17.1 and 20.6, 19.7 and 21.9, 131072 22.8 and 21.7; 127 trees 42.7 and 60.2 over 65536, 78.0 and 79.3 over 131072, 128
// 42.3 and 60.9, 78.0 and 81.3.  So it holds for 16 to 64 sequences of 98304 tokens on; what lies nearer to it loses up to 17 us.
bool in_rounds(int batch, int vocab) { return batch < 128 && vocab >= 65536; }

}  // namespace

size_t verify_scratch_bytes(int batch, int, int vocab) {
  Scratch x;
  return in_rounds(batch, vocab) ? scratch_of(x, nullptr, batch) : 0;
}

int launch_verify(const treekv_verify_args& a, hipStream_t s) {
  const int rounds = !in_rounds(a.batch, a.vocab) ? 0 : a.draft ? ROUNDS : 1;
  Scratch x;
  scratch_of(x, (char*)a.scratch, a.batch);
  auto part = a.dtype == TREEKV_F32 ? verify_part_kernel<float> : verify_part_kernel<uint16_t>;
  auto last = a.dtype == TREEKV_F32 ? verify_kernel<float> : verify_kernel<uint16_t>;
  for (int i = 0; i < rounds; ++i) hipLaunchKernelGGL(part, dim3(a.batch * VF_WAVES), dim3(PART_THREADS), 0, s, a, x, i);
  hipLaunchKernelGGL(last, dim3(a.batch), dim3(VF_THREADS), 0, s, a, x, rounds);
  return finish_launch();
}

}  // namespace tkv
