// Microscaled 4-bit codes (E2M1 with one E8M0 scale per 32 channels), the norm before a
// projection, and the product of such codes: launchers and device helpers.
#pragma once

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
size_t mx_gemm_workspace(int64_t M, int64_t N, int64_t K);
hipError_t launch_mx_gemm(const MxGemmArgs &g, void *ws, hipStream_t s);

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

#endif  // __HIPCC__

}  // namespace fq
