// Microscaled 4-bit codes (E2M1 with one E8M0 scale per 32 channels), the norm before a
// projection, and the product of such codes: launchers and device helpers.
#pragma once

#include "fq_codes.hpp"
#include "fq_device.hpp"

namespace fq {

// Codes: nibbles [M, K/2], channel 2i in the low half of byte i.  Scales: bytes [K/128][M][4],
// the four blocks of a row's 128-channel step adjacent, so that a tile's scales of one step
// are one run and a lane of the product takes its block's byte out of one word.
__host__ __device__ inline int64_t mx_scale_word(int64_t row, int64_t M, int step) { return (int64_t)step * M + row; }

struct MxQuantArgs {
  const void *x;  // bf16 or fp32 [M, ldx]
  bool x_is_f32;
  int64_t ldx;
  const float *pre, *post;  // [K] or NULL
  int64_t M;
  int K, b;
  float cb;
  uint8_t *codes, *scales;
};
hipError_t launch_mx_quant(const MxQuantArgs &a, hipStream_t s);
inline int log2_of(int b) {
  int k = 0;
  while ((1 << k) < b) ++k;
  return k;
}

// Output of the norm: eq. (5) codes (kOutNibble, kOutInt8) or kOutMx.
constexpr int kOutMx = 3;
struct NormArgs {
  const void *x;  // bf16 [M, ldx]
  int64_t ldx;
  const void *residual;  // bf16 [M, ldr] or NULL
  int64_t ldr;
  const float *weight, *post;  // [K]; post may be NULL
  float eps;
  int64_t M;
  int K, b;
  float clip_ratio, cb;
  void *sum;  // bf16 [M, lds] or NULL
  int64_t lds;
  int out_fmt;
  uint8_t *codes;
  float *delta;     // kOutNibble, kOutInt8
  uint8_t *scales;  // kOutMx
};
hipError_t launch_norm_quant(const NormArgs &a, hipStream_t s);

// Codes as bf16 values.  scale: fp32 [M] (bits 4 or 8) or bytes (bits 0: microscaled).
hipError_t launch_read_codes(const uint8_t *codes, const void *scale, int64_t M, int K, int bits, uint16_t *values,
                             int64_t ldv, hipStream_t s);
// Nibbles [N, K/2] to 16 x 128 tiles and back.
hipError_t launch_mx_pack(const uint8_t *from, int64_t N, int K, bool unpack, uint8_t *to, hipStream_t s);

struct MxGemmArgs {
  const uint8_t *a, *a_scale;  // codes [M, K/2], scales [K/128][M][4]
  const uint8_t *w, *w_scale;  // tiles, scales [K/128][N][4]
  const float *bias;
  uint16_t *y;
  int64_t ldy;
  int64_t M, N;
  int K;
};
// How a product of these sizes is launched (mx_plan).
struct MxPlan {
  int stream, tile, splits;  // one of stream and tile is -1
  bool token;                // the projection in one launch
};
MxPlan mx_plan(int64_t M, int64_t N, int64_t K);
inline size_t mx_gemm_workspace(const MxPlan &p, int64_t M, int64_t N) {
  return p.splits > 1 ? (size_t)p.splits * (size_t)M * (size_t)N * 4 : 0;
}
hipError_t launch_mx_gemm(const MxGemmArgs &g, const MxPlan &p, void *ws, hipStream_t s);
// Rounding and product in one launch (p.token), the same outputs.  g.a, g.a_scale and q's outputs are not used.
hipError_t launch_mx_token(const MxQuantArgs &q, const MxGemmArgs &g, const MxPlan &p, hipStream_t s);

#if defined(__HIPCC__)

// Scale byte of a block: floor(log2 amax) - 2, biased by 127, at least 0 (an empty block too);
// 255 where amax is infinite or NaN.
__device__ __forceinline__ uint32_t mx_scale_byte(float amax) {
  const uint32_t e = __float_as_uint(amax) >> 23;
  return e == 255 ? 255u : (uint32_t)max((int)e - 2, 0);
}
// 2^(byte - 127); byte 0 is subnormal.
__device__ __forceinline__ float mx_scale_value(uint32_t byte) {
  return __uint_as_float(byte ? byte << 23 : 0x00400000u);
}
// max |v| that a NaN passes through (v_maximum3_f32).
__device__ __forceinline__ float abs_maximum(float m, float a, float b) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_elementwise_maximum(__builtin_elementwise_maximum(m, __builtin_fabsf(a)), __builtin_fabsf(b));
#else
  return m + a + b;
#endif
}
__device__ __forceinline__ float maximum(float a, float b) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_elementwise_maximum(a, b);
#else
  return a + b;
#endif
}

// 16 values over the scale to 16 codes, 8 bytes in channel order: v_cvt_scalef32_pk_fp4_f32
// rounds v / 2^(byte - 127) to nearest, ties to even, and saturates at 6 (checked against that
// rule for every scale, at ties and at their neighbours).  A block with the scale NaN has codes 0.
__device__ __forceinline__ uint2 mx_pack16(const float (&v)[16], uint32_t byte) {
  uint2 r = make_uint2(0, 0);
#if defined(__HIP_DEVICE_COMPILE__)
  const float s = mx_scale_value(byte);
#define FQ_PK(w, i, sel) w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[i], v[i + 1], s, sel)
  FQ_PK(r.x, 0, 0); FQ_PK(r.x, 2, 1); FQ_PK(r.x, 4, 2); FQ_PK(r.x, 6, 3);
  FQ_PK(r.y, 8, 0); FQ_PK(r.y, 10, 1); FQ_PK(r.y, 12, 2); FQ_PK(r.y, 14, 3);
#undef FQ_PK
#endif
  if (byte == 255) r = make_uint2(0, 0);
  return r;
}

// Chunk of lane tau of a 16-lane group: bits 2 and 3 swapped, so that the stage h = 64 is a DPP
// rotation by 8 lanes and only h = 128 needs the LDS crossbar (as the prologue's kernel).
__device__ __forceinline__ int mx_chunk(int tau) { return (tau & ~12) | ((tau & 4) << 1) | ((tau & 8) >> 1); }

// The unnormalized block Hadamard of 2^log2b channels (uniform), lanes holding chunks mx_chunk(tau).
// The values come out times the sign that it returns.
template <int CPT>
__device__ __forceinline__ float mx_transform(float (&v)[CPT][16], int log2b, int tau) {
#pragma unroll
  for (int c = 0; c < CPT; ++c) {
    if (log2b > 0) chunk_stage<1>(v[c]);
    if (log2b > 1) chunk_stage<2>(v[c]);
    if (log2b > 2) chunk_stage<4>(v[c]);
    if (log2b > 3) chunk_stage<8>(v[c]);
  }
  int mask = 0;
  if (log2b > 4) lane_stage<1, CPT>(v, tau), mask |= 1;
  if (log2b > 5) lane_stage<2, CPT>(v, tau), mask |= 2;
  if (log2b > 6) lane_stage<8, CPT>(v, tau), mask |= 8;
  if (log2b > 7) lane_stage<4, CPT>(v, tau), mask |= 4;
  return (__builtin_popcount(tau & mask) & 1) ? -1.0f : 1.0f;
}

__device__ __forceinline__ void load_mult(const float *m, int chunk, float4 (&f)[4]) {
  const float4 *p = reinterpret_cast<const float4 *>(m) + (int64_t)chunk * 4;
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = p[i];
}

// max |v| of a block's 32 channels: the chunk's 16 and those of the lane next to it.
__device__ __forceinline__ float block_max(const float (&v)[16]) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 16; i += 2) m = abs_maximum(m, v[i], v[i + 1]);
  return maximum(m, lane_xor<1>(m));
}

// The four scale bytes of a 128-channel step, in all of its eight lanes (chunk bits 1, 2 are lane bits
// 1, 3).
__device__ __forceinline__ uint32_t step_scales(uint32_t byte, int tau) {
  uint32_t w = byte << (8 * (((tau >> 1) & 1) | ((tau >> 2) & 2)));
  w |= __float_as_uint(lane_xor<2>(__uint_as_float(w)));
  w |= __float_as_uint(lane_xor<8>(__uint_as_float(w)));
  return w;
}

#endif  // __HIPCC__

}  // namespace fq
