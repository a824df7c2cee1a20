// treekv_tree_verify: the accepted path of a drafted tree and the token that follows it, for gfx950.
//
// The nodes come after their parents, so one walk over them in order meets the children of the last accepted token, and after
// an acceptance the new one's.  With P the target's row there and Q the drafter's, k refusals leave
//   P_k = max(P - c_k Q, 0) / W_k,   W_k = sum of max(P - c_k Q, 0),   c_1 = 1,  c_k+1 = c_k + W_k
// (each step subtracts Q from what the last one made sum to 1, that is, W_k times Q from what it was made of), so a refusal is
// one pass over two rows, whatever came before it, and the next child is accepted if u Q(x) W_k < max(P(x) - c_k Q(x), 0).
// Sums are in double: 2^24 terms leave 2^-29 of a step of fp32, so whether a token is accepted or follows does not depend on
// their order but within that.
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
  // the values of one 16-byte piece; those that are no part of the row are 0
  __device__ void piece(int j, double (&y)[EPL]) const {
    const int x0 = j * EPL - skew;
    float a[EPL], b[EPL];
    if (x0 >= 0 && x0 + EPL <= vocab) {
      Storage<T>::widen(*reinterpret_cast<const uint4*>(p + x0), a);
      if (q) Storage<T>::widen(*reinterpret_cast<const uint4*>(q + x0), b);
    } else {
#pragma unroll
      for (int e = 0; e < EPL; ++e) {
        const bool in = x0 + e >= 0 && x0 + e < vocab;
        a[e] = in ? value_at(p, x0 + e) : 0.f;
        b[e] = in && q ? value_at(q, x0 + e) : 0.f;
      }
    }
#pragma unroll
    for (int e = 0; e < EPL; ++e) y[e] = q ? fmax(positive(a[e]) - c * positive(b[e]), 0.0) : positive(a[e]);
    for (int i = 0; i < n_out; ++i) {
      const int e0 = out[i] - x0;
      if (e0 >= 0 && e0 < EPL)
#pragma unroll
        for (int e = 0; e < EPL; ++e)
          if (e == e0) y[e] = 0.0;
    }
  }
};

__device__ inline double wave_sum(double v) {
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) v += __shfl_xor(v, x, 64);
  return v;
}
// Pieces [lo, hi) summed by the wave.
template <typename T>
__device__ inline double sum_pieces(const Left<T>& l, int lo, int hi) {
  double sum = 0.0;
  for (int j = lo + (int)(threadIdx.x & 63); j < hi; j += 64) {
    double y[Left<T>::EPL];
    l.piece(j, y);
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

template <typename T>
__global__ __launch_bounds__(VF_THREADS) void verify_kernel(treekv_verify_args a) {
  __shared__ double sm[VF_WAVES];
  __shared__ int parent[TREEKV_TREE_MAX_NODES], token[TREEKV_TREE_MAX_NODES], out[TREEKV_TREE_MAX_NODES], found;
  __shared__ float uniform[TREEKV_TREE_MAX_NODES + 1];
  const int b = blockIdx.x, tid = threadIdx.x, n = a.n, V = a.vocab;
  if (tid < n) {
    parent[tid] = a.parents[(size_t)b * n + tid];
    token[tid] = a.tokens[(size_t)b * n + tid];
  }
  if (tid <= n) uniform[tid] = a.uniforms[(size_t)b * (n + 1) + tid];
  __syncthreads();
  Left<T> l;
  l.vocab = V;
  l.out = out;
  int at = -1, len = 0;
  double W = 1.0;
  bool summed = false;               // sm holds the sums of what is left now
  auto enter = [&](int node) {       // the rows after `node`
    const size_t row = ((size_t)b * (n + 1) + node + 1) * V;
    l.p = (const T*)a.target + row;
    l.q = nullptr;
    l.c = 0.0;
    l.skew = (int)(row % Left<T>::EPL);
    l.n_out = 0;
    W = 1.0;
    summed = false;
  };
  enter(-1);
  const T* draft = nullptr;
  for (int i = 0; i < n; ++i) {
    if (parent[i] != at) continue;
    const int x = token[i];
    if (x < 0 || x >= V) continue;
    const double u = uniform[i], p = positive(value_at(l.p, x));
    bool accepted;
    if (a.draft) {
      draft = (const T*)a.draft + (l.p - (const T*)a.target);
      const double q = positive(value_at(draft, x));
      accepted = u * q * W < fmax(p - l.c * q, 0.0);
    } else {
      bool gone = false;
      for (int j = 0; j < l.n_out; ++j) gone |= out[j] == x;
      accepted = u * W < (gone ? 0.0 : p);
      if (!accepted && !gone) {
        W = fmax(W - p, 0.0);
        __syncthreads();
        if (tid == 0) out[l.n_out] = x;
        __syncthreads();
        ++l.n_out;
      }
    }
    if (accepted) {
      if (tid == 0) a.path[(size_t)b * n + len] = i;
      ++len;
      at = i;
      enter(at);
    } else if (a.draft) {
      Left<T> next = l;
      next.q = draft;
      next.c = l.c + W;
      const double left = sum_parts(next, 0, next.pieces(), sm);
      summed = left > 0.0;
      if (summed) {
        l = next;
        W = left;
      }
    }
  }
  double total = W;
  if (!summed) total = sum_parts(l, 0, l.pieces(), sm);
  if (!(total > 0.0) && (l.q || l.n_out)) {
    enter(at);
    total = sum_parts(l, 0, l.pieces(), sm);
  }
  const int next = draw(l, (double)uniform[n], total, sm, &found);
  for (int i = len + tid; i < n; i += VF_THREADS) a.path[(size_t)b * n + i] = -1;
  if (tid == 0) {
    a.path_len[b] = len;
    a.next_token[b] = next;
  }
}

}  // namespace

size_t verify_scratch_bytes(int, int, int) { return 0; }

int launch_verify(const treekv_verify_args& a, hipStream_t s) {
  if (a.dtype == TREEKV_F32) hipLaunchKernelGGL(verify_kernel<float>, dim3(a.batch), dim3(VF_THREADS), 0, s, a);
  else hipLaunchKernelGGL(verify_kernel<uint16_t>, dim3(a.batch), dim3(VF_THREADS), 0, s, a);
  return finish_launch();
}

}  // namespace tkv
