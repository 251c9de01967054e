// Device helpers shared by the attention kernels: bf16 matrix products, code conversion, the
// rows and keys of a workgroup, and what a row's result is written to.
//
// Both kernels compute S^T = K Q^T and O^T = V^T P^T, so that a lane's accumulators of S^T all
// belong to one query row (the instruction's column): the softmax of a row is in-lane but for one
// exchange between the lanes that share the row, and P^T is already in the operand order of the
// second product.  The order of tokens along a tile is chosen so that a lane's accumulators are
// consecutive tokens of one 16-token group, hence under one scale of the cache.
#pragma once

#include <cfloat>

#include "fq_attn.hpp"
#include "fq_device.hpp"

namespace fq {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

// Accumulators: C[row m][column n] of lane l: 16 x 16: n = l % 16, m = 4 (l / 16) + r;
// 32 x 32: n = l % 32, m = 8 (r / 4) + 4 (l / 32) + r % 4.  Operands: row (column) l % 16 or
// l % 32, and 8 consecutive k per lane group l / 16 or l / 32.
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Two floats to packed bf16, round to nearest even.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const f32x2 v = {a, b};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
}

// Sum of two packed bf16 values and an fp32 one.
__device__ __forceinline__ float add_pair(uint32_t pair, float sum) {
#if defined(__HIP_DEVICE_COMPILE__)
  const bf16x2 one = {(__bf16)1.0f, (__bf16)1.0f};
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), one, sum, false);
#else
  return sum;
#endif
}

// Four int8 codes -> four bf16 (exact: |code| <= 128 has at most 8 significant bits): the float of
// a code holds it in its upper half.
__device__ __forceinline__ uint2 codes_to_bf16(uint32_t w) {
  const uint32_t f0 = __float_as_uint((float)(int8_t)w), f1 = __float_as_uint((float)(int8_t)(w >> 8));
  const uint32_t f2 = __float_as_uint((float)(int8_t)(w >> 16)), f3 = __float_as_uint((float)((int32_t)w >> 24));
  return make_uint2(__builtin_amdgcn_perm(f1, f0, 0x07060302u), __builtin_amdgcn_perm(f3, f2, 0x07060302u));
}
__device__ __forceinline__ uint4 codes8_to_bf16(uint32_t a, uint32_t b) {
  const uint2 x = codes_to_bf16(a), y = codes_to_bf16(b);
  return make_uint4(x.x, x.y, y.x, y.y);
}

// Value of lane l ^ 32 (l ^ 16) combined by max or sum: the swaps exchange halves of two registers,
// which gives both sides of the pair to both lanes.
template <typename F>
__device__ __forceinline__ float across32(float v, F f) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
  return v;
#endif
}
template <typename F>
__device__ __forceinline__ float across16(float v, F f) {
#if defined(__HIP_DEVICE_COMPILE__)
  const uint32_t u = __float_as_uint(v);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
#else
  return v;
#endif
}
__device__ __forceinline__ float maxf(float a, float b) { return __builtin_fmaxf(a, b); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Transposing LDS read: within 16 lanes, lane i gets element i % 4 of the 8-byte pieces that
// lanes i / 4, i / 4 + 4, i / 4 + 8, i / 4 + 12 address; with piece p at token p / 4, channels
// 4 (p % 4) .., lane i has channel i of four tokens.
__device__ __forceinline__ uint2 lds_read_transposed(const void *p) {
#if defined(__HIP_DEVICE_COMPILE__)
  typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
  const s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(p));
  return __builtin_bit_cast(uint2, v);
#else
  return make_uint2(0, 0);
#endif
}

// The rows of one sequence: row r of a key head is query i = r / G, head h G + r % G.  Counts and
// places of tokens are below 2^30, rows of a key head below 2^31.
struct Rows {
  int64_t q0;   // first row of the sequence in q and out
  int n;        // queries
  int keys;     // keys there are
  int back;     // causal: query i sees keys up to back + i
  bool causal;
  // keys that query i sees: [0, end(i))
  __device__ __forceinline__ int end(int i) const {
    if (!causal) return keys;
    const int e = back + i + 1;
    return e < 0 ? 0 : e < keys ? e : keys;
  }
};
template <bool CACHED>
__device__ __forceinline__ Rows sequence_queries(const AttnArgs &a, int64_t s) {
  Rows r;
  const int max_new = (int)a.max_new, max_kv = (int)a.max_kv;
  if constexpr (CACHED) {
    const int T = (int)a.T;
    int q0 = a.b.q_start[s], q1 = a.b.q_start[s + 1];
    q0 = q0 < 0 ? 0 : q0 > T ? T : q0;
    q1 = q1 < q0 ? q0 : q1 > T ? T : q1;
    const int len = a.b.kv_len[s] < 0 ? 0 : a.b.kv_len[s];
    r.q0 = q0;
    r.n = q1 - q0 < max_new ? q1 - q0 : max_new;
    r.keys = len < max_kv ? len : max_kv;
    r.back = len - (q1 - q0);
    r.causal = a.causal != 0;
  } else {
    r.q0 = s * a.max_new;
    r.n = max_new;
    r.keys = max_kv;
    if (a.kv_len) {
      const int len = a.kv_len[s];
      r.keys = len < 0 ? 0 : len < max_kv ? len : max_kv;
    }
    r.back = 0;
    r.causal = false;
  }
  return r;
}

__device__ __forceinline__ int clamp_page(int p, int64_t pages) {
  return p < 0 ? 0 : p >= pages ? (int)(pages - 1) : p;
}
__device__ __forceinline__ int64_t cache_page(const AttnArgs &a, int64_t s, int64_t w) {
  return clamp_page(a.b.pt[s * a.b.width + w], a.c.pages);
}

// How a call's tokens are split: `splits` ranges of `chunk` tokens; with more than one, fp32
// partial results o [splits][seqs][Hk][max_new G][D] and (maximum, sum) ml [splits][...] go to the
// workspace and a second kernel joins them.
struct Split {
  int chunk;
  int splits;
  float *o;
  float2 *ml;
};

}  // namespace fq
