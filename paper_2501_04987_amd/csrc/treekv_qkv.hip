// treekv_qkv_prepare: the heads of q and k normalised and turned, v copied, out of the rows of a projection.
//
//   y = R(position) (x / sqrt(mean(x^2) + eps) * w),   R: plane i turned by position * inv_freq[i]
//
// A head is D elements in D / 8 (bf16) or D / 4 (fp32) lanes of 16 bytes; the mean of squares is one sum over those lanes,
// the two dimensions of a plane lie in one lane (2i, 2i+1) or, for halves, rotary_dim / 2 dimensions apart in the same head:
// one exchange of lanes, since rotary_dim is a multiple of 16.  A token's angles are formed once per workgroup, in double (a
// position of a million times a frequency near 1 leaves 2^-33 of a turn), and reduced to a turn.  With fp32 storage their sines
// and cosines are taken in double too and rounded once; for bf16 the reduced angle is rounded to fp32 first, which moves them by
// 2^-23 at most, where the result's half step is 2^-9.
// Bound by memory: every head once in and once out.

#include "treekv_internal.h"

namespace tkv {

namespace {

constexpr int QKV_THREADS = 256;

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;

__device__ inline uint4 narrow(const float (&y)[8], uint16_t) {
  unsigned w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x2_t v = {y[2 * i], y[2 * i + 1]};
    w[i] = __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2_t));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ inline uint4 narrow(const float (&y)[4], float) {
  return make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
}

// Sine of h half turns, |h| < 2, rounded once: reduced to a quarter turn either way (exactly) and from there by its power series,
// whose first term left out is 2^-45 of it (x^18 / 19!).  (The library's double functions, good for all 53 bits, take 44
// registers more, and with fewer workgroups side by side 16384 tokens of 48 heads x 128 take 167 us in place of 150, as long as
// with angles rounded to fp32 first.)
__device__ inline float sine(double h) {
  const double whole = rint(h), x = (h - whole) * 3.14159265358979323846, y = x * x;
  double s = 1.0 / 355687428096000.0;                // 17!
  s = fma(s, y, -1.0 / 1307674368000.0);
  s = fma(s, y, 1.0 / 6227020800.0);
  s = fma(s, y, -1.0 / 39916800.0);
  s = fma(s, y, 1.0 / 362880.0);
  s = fma(s, y, -1.0 / 5040.0);
  s = fma(s, y, 1.0 / 120.0);
  s = fma(s, y, -1.0 / 6.0);
  const float r = (float)fma(s * y, x, x);
  return (int)whole & 1 ? -r : r;
}

// What happens to one 16-byte piece of a head (`part` of it; the lanes of a head lie side by side).  Returns the piece of the
// output this lane writes.
template <typename T, int D>
__device__ inline int work_piece(const treekv_qkv_args& a, const float2* cs, bool turn, bool norm, const uint4& wraw, int part, uint4& raw) {
  constexpr int EPL = Storage<T>::EPL, LPR = D / EPL;
  const int half = a.rotary_dim / 2;
  float x[EPL];
  Storage<T>::widen(raw, x);
  if (norm) {
    float sum = 0.f, w[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) sum = fmaf(x[e], x[e], sum);
    const float inv = rsqrtf(group_sum<LPR>(sum) * (1.0f / D) + a.eps);
    Storage<T>::widen(wraw, w);
#pragma unroll
    for (int e = 0; e < EPL; ++e) x[e] = x[e] * inv * w[e];
  }
  int to_part = part;
  if (turn && (a.flags & TREEKV_ROPE_HALVES) && half > 0) {
    // lanes of the first half hold the first dimensions of planes part * EPL .., those of the second half the second ones
    const int lanes = half / EPL;
    const bool turned = part < 2 * lanes, second = part >= lanes;
    const int other = turned ? (second ? -lanes : lanes) : 0, plane = (second ? part - lanes : part) * EPL;
    float ya[EPL], yb[EPL];
#pragma unroll
    for (int e = 0; e < EPL; ++e) {
      const float o = __shfl(x[e], (threadIdx.x & 63) + other, 64);
      const float2 t = a.positions && turned ? cs[plane + e] : make_float2(1.f, 0.f);
      const float p0 = second ? o : x[e], p1 = second ? x[e] : o;
      ya[e] = a.positions ? p0 * t.x - p1 * t.y : p0;        // (not turned at all: an infinity times 0 would be a NaN)
      yb[e] = a.positions ? p0 * t.y + p1 * t.x : p1;
    }
    if (turned) {
      if (a.flags & TREEKV_ROPE_TO_PLANES) {
        // planes plane .. plane + EPL - 1 are 2 EPL output dimensions; this lane writes the first or the second EPL of them
        to_part = 2 * (plane / EPL) + (second ? 1 : 0);
#pragma unroll
        for (int e = 0; e < EPL / 2; ++e) {
          x[2 * e] = second ? ya[EPL / 2 + e] : ya[e];
          x[2 * e + 1] = second ? yb[EPL / 2 + e] : yb[e];
        }
      } else {
#pragma unroll
        for (int e = 0; e < EPL; ++e) x[e] = second ? yb[e] : ya[e];
      }
    }
  } else if (turn && a.positions && part * EPL < a.rotary_dim) {
#pragma unroll
    for (int e = 0; e < EPL; e += 2) {
      const float2 t = cs[(part * EPL + e) / 2];
      const float p0 = x[e], p1 = x[e + 1];
      x[e] = p0 * t.x - p1 * t.y;
      x[e + 1] = p0 * t.y + p1 * t.x;
    }
  }
  raw = narrow(x, T());
  return to_part;
}

// A workgroup takes ITER heads per lane group of one token (a run of its q, k and v heads), all requested before the angles are
// formed.  ITER = 4 forms the angles once per token of 64 heads and keeps four loads in flight: 32768 tokens of 48 heads x 128
// 164 -> 153 us; a few tokens' heads are spread over more workgroups instead (one token of 96 heads 2.9 us).  976 tokens take
// 8.3 us for 24 MB: a workgroup's only token waits for its position, its angles in double and a barrier before it is stored.
template <typename T, int D, int ITER, bool STREAM>
__global__ __launch_bounds__(QKV_THREADS, 6) void qkv_kernel(treekv_qkv_args a, int chunks) {
  constexpr int LPR = D / Storage<T>::EPL, ROWS = QKV_THREADS / LPR;
  __shared__ float2 cs[D / 2];
  const int tid = threadIdx.x, part = tid % LPR;
  const int nq = a.q ? a.q_heads : 0, nk = a.k ? a.kv_heads : 0, nv = a.v ? a.kv_heads : 0;
  const long long items = (long long)a.tokens * chunks;
  for (long long item = blockIdx.x; item < items; item += gridDim.x) {
    const int token = (int)(item / chunks), first = (int)(item % chunks) * (ROWS * ITER) + tid / LPR;
    // a head's source, destination and what happens to it
    auto kind_of = [&](int row) { return row < nq ? 0 : row < nq + nk ? 1 : 2; };
    auto head_of = [&](int row) { return row < nq ? row : row < nq + nk ? row - nq : row - nq - nk; };
    uint4 raw[ITER], w[ITER];
#pragma unroll
    for (int x = 0; x < ITER; ++x) {
      const int row = first + x * ROWS, kind = kind_of(row), head = head_of(row);
      raw[x] = w[x] = make_uint4(0, 0, 0, 0);
      if (row < nq + nk + nv) {
        const T* src = (const T*)(kind == 0 ? a.q : kind == 1 ? a.k : a.v) +
                       (long long)token * (kind == 0 ? a.q_stride : kind == 1 ? a.k_stride : a.v_stride) + (long long)head * D;
        const void* weight = kind == 0 ? a.q_weight : kind == 1 ? a.k_weight : nullptr;
        raw[x] = reinterpret_cast<const uint4*>(src)[part];
        if (weight) w[x] = reinterpret_cast<const uint4*>(weight)[part];
      }
    }
    // half turns, less whole turns (the fraction is exact, whatever their number)
    auto half_turns = [&](int plane) {
      const double turns = (double)a.positions[token] * a.inv_freq[plane] * 0.15915494309189533577;
      return 2.0 * (turns - rint(turns));
    };
    if constexpr (sizeof(T) == 4) {                  // a lane for each cosine, which is a sine a quarter turn on, and each sine
      if (a.positions && tid < a.rotary_dim) (&cs[tid >> 1].x)[tid & 1] = sine(half_turns(tid >> 1) + (tid & 1 ? 0.0 : 0.5));
    } else if (a.positions && tid < a.rotary_dim / 2) {
      float s, c;
      sincospif((float)half_turns(tid), &s, &c);
      cs[tid] = make_float2(c, s);
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < ITER; ++x) {
      const int row = first + x * ROWS, kind = kind_of(row), head = head_of(row);
      int to_part = part;
      if (kind < 2) to_part = work_piece<T, D>(a, cs, true, kind == 0 ? a.q_weight != nullptr : a.k_weight != nullptr, w[x], part, raw[x]);
      if (row < nq + nk + nv) {
        T* dst = (T*)(kind == 0 ? a.q_out : kind == 1 ? a.k_out : a.v_out) +
                 ((long long)token * (kind == 0 ? a.q_heads : a.kv_heads) + head) * D;
        store16<STREAM>(reinterpret_cast<uint4*>(dst) + to_part, raw[x]);
      }
    }
    __syncthreads();                                 // the next item's angles
  }
}

template <typename T, int D>
int launch_qkv_d(const treekv_qkv_args& a, hipStream_t s) {
  constexpr int ROWS = QKV_THREADS / (D / Storage<T>::EPL);
  const int rows = (a.q ? a.q_heads : 0) + (a.k ? a.kv_heads : 0) + (a.v ? a.kv_heads : 0);
  const bool few = (long long)a.tokens * ((rows + ROWS - 1) / ROWS) <= 512;          // two workgroups a compute unit
  const int per = few ? ROWS : 4 * ROWS, chunks = (rows + per - 1) / per;
  const long long items = (long long)a.tokens * chunks, most = 1 << 20;
  // (32768 tokens of 48 heads x 128: 145 us so on the card where it took 153 through the caches; 145-161 from card to card,
  // 5.0 to 5.6 TB/s in and out)
  const bool stream = (size_t)a.tokens * rows * D * sizeof(T) > STREAM_BYTES;
  auto kernel = few ? qkv_kernel<T, D, 1, false> : stream ? qkv_kernel<T, D, 4, true> : qkv_kernel<T, D, 4, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)(items < most ? items : most)), dim3(QKV_THREADS), 0, s, a, chunks);
  return finish_launch();
}

}  // namespace

int launch_qkv(const treekv_qkv_args& a, hipStream_t s) {
  if (a.dtype == TREEKV_F32) return a.head_dim == 128 ? launch_qkv_d<float, 128>(a, s) : launch_qkv_d<float, 64>(a, s);
  return a.head_dim == 128 ? launch_qkv_d<uint16_t, 128>(a, s) : launch_qkv_d<uint16_t, 64>(a, s);
}

}  // namespace tkv
