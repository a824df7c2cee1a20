// Operands of the matrix instructions as the attention kernels that read K and V straight from memory use them.
//
//   S^T = K Q^T      A operand: lane (r, g) = (lane % 16, lane / 16) holds 16 bytes of K row r: the row's pieces 4 s + g in step s
//   O^T += V^T P^T   a lane's logits are columns 4 g + i (+ 16) of row r, which is the B operand as it lies.  The A operand
//                    wants those columns of one dimension; the lane loads 16 bytes (8 at head_dim 64) of each of those rows,
//                    that is, its columns of dimensions r * D/16 .. + D/16 - 1, and one byte permutation per pair of columns
//                    makes the operand of each dimension.  The lane's sums are then of row r, dimensions g * D/4 .. + D/4 - 1.
#pragma once

#include "treekv_internal.h"

namespace tkv {

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(16))) float f32x16_t;

constexpr float REF_NONE = -3.0e38f;               // reference of a row that has seen nothing: below every logit, and finite, so that exp2(-inf - it) = 0
constexpr float LN2 = 0.6931471805599453f, LOG2E = 1.4426950408889634f;

__device__ inline f32x4_t mfma_bf16(const uint4& a, const uint4& b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ inline f32x16_t mfma_wide(const uint4& a, const uint4& b, f32x16_t c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}
__device__ inline float row_max(float v) {          // over the four lanes, 16 apart, of a row
  v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
__device__ inline float row_sum(float v) {
  v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}

// 8 and 16 bytes; ONCE: past the caches, which nobody asks for them again.
template <bool ONCE>
__device__ inline uint4 load16(const void* p) {
  typedef unsigned v4u __attribute__((ext_vector_type(4)));
  if constexpr (ONCE) return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const v4u*>(p)));
  else return *reinterpret_cast<const uint4*>(p);
}
template <bool ONCE>
__device__ inline uint2 load8(const void* p) {
  typedef unsigned v2u __attribute__((ext_vector_type(2)));
  if constexpr (ONCE) return __builtin_bit_cast(uint2, __builtin_nontemporal_load(reinterpret_cast<const v2u*>(p)));
  else return *reinterpret_cast<const uint2*>(p);
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
  template <bool ONCE = false>
  __device__ static inline void load_v(Values& v, int j, const char* base, unsigned row) {
    if constexpr (D == 128) v.x[j] = load16<ONCE>(base + row);
    else {
      const uint2 r = load8<ONCE>(base + row);
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
  template <bool ONCE = false>
  __device__ static inline void load_v(Values& v, int j, const char* base, unsigned row) {
#pragma unroll
    for (int e = 0; e < DPL; e += 4) {
      const float4 r = __builtin_bit_cast(float4, load16<ONCE>(base + row + e * 4));
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

}  // namespace

}  // namespace tkv
