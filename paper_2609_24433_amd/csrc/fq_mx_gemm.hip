// Product of microscaled 4-bit codes: y = bf16(sum over blocks 2^(ea + ew - 254) sum a w + bias) on the
// matrix instructions that take E2M1 operands with a scale byte per lane.
#include "fq_launch.hpp"
#include "fq_mx.hpp"

namespace fq {

namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));

// 16 x 16 x 128: lane l holds row (or column) l % 16 and block l / 16, 32 codes in four words (a format
// selector of 4 is E2M1), its scale in the low byte of sa (sb).
__device__ __forceinline__ v4f mfma_mx_16(const v4i &a, int sa, const v4i &b, int sb, v4f c) {
#if defined(__HIP_DEVICE_COMPILE__)
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v8i{a.x, a.y, a.z, a.w, 0, 0, 0, 0},
                                                          v8i{b.x, b.y, b.z, b.w, 0, 0, 0, 0}, c, 4, 4, 0, sa, 0, sb);
#else
  return c;
#endif
}

// One wave per 16 columns and 16 MT rows, operands straight from memory.
template <int MT>
__global__ __launch_bounds__(256) void mx_gemm_rows_kernel(MxGemmArgs p) {
  const int lane = threadIdx.x & 63, r16 = lane & 15, g = lane >> 4;
  const uint32_t cols = (uint32_t)((p.N / 16 + 3) / 4), rb = blockIdx.x / cols;
  const int64_t nb = (int64_t)(blockIdx.x - rb * cols) * 4 + (threadIdx.x >> 6);
  if (nb * 16 >= p.N) return;
  const int ktot = p.K / kTileK;
  const int64_t m0 = (int64_t)rb * 16 * MT;
  const uint8_t *w = p.w + nb * ktot * 1024 + lane * 16;
  const uint32_t *ws = reinterpret_cast<const uint32_t *>(p.w_scale) + nb * 16 + r16;
  const uint8_t *a[MT];
  const uint32_t *as[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int64_t row = m0 + 16 * t + r16 < p.M ? m0 + 16 * t + r16 : p.M - 1;
    a[t] = p.a + row * (p.K / 2) + g * 16;
    as[t] = reinterpret_cast<const uint32_t *>(p.a_scale) + row;
  }
  v4f acc[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) acc[t] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll 2
  for (int ks = 0; ks < ktot; ++ks) {
    const v4i b = *reinterpret_cast<const v4i *>(w + (int64_t)ks * 1024);
    const int sb = (int)(ws[(int64_t)ks * p.N] >> (8 * g));
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      const v4i x = *reinterpret_cast<const v4i *>(a[t] + ks * 64);
      acc[t] = mfma_mx_16(x, (int)(as[t][(int64_t)ks * p.M] >> (8 * g)), b, sb, acc[t]);
    }
  }
  const float bias = p.bias ? p.bias[nb * 16 + r16] : 0.0f;
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t m = m0 + 16 * t + 4 * g + i;
      if (m < p.M) p.y[m * p.ldy + nb * 16 + r16] = (uint16_t)f32_to_bf16(acc[t][i] + bias);
    }
}

}  // namespace

size_t mx_gemm_workspace(int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_mx_gemm(const MxGemmArgs &g, void *, hipStream_t s) {
  const int rows = g.M <= 16 ? 16 : 64;
  const int64_t grid = (g.N / 16 + 3) / 4 * ((g.M + rows - 1) / rows);  // at most 2^40 outputs: fits 31 bits
  if (rows == 16) hipLaunchKernelGGL(mx_gemm_rows_kernel<1>, dim3((unsigned)grid), dim3(256), 0, s, g);
  else hipLaunchKernelGGL(mx_gemm_rows_kernel<4>, dim3((unsigned)grid), dim3(256), 0, s, g);
  return hipGetLastError();
}

}  // namespace fq
