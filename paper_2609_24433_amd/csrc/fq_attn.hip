// Attention over the 8-bit paged cache and over bf16 states of another length.
#include "fq_attn.hpp"
#include "fq_device.hpp"

namespace fq {
namespace {

// One query row of one head a wave: 64 keys a step, one a lane, under a running maximum and sum;
// then the values, D/64 channels a lane.
template <bool CACHED>
__global__ __launch_bounds__(64) void attention_row_kernel(AttnArgs a) {
  __shared__ float qs[256];
  __shared__ float ps[64];
  const int D = a.D, lane = threadIdx.x;
  const int hq = blockIdx.x % a.Hq, h = hq / (a.Hq / a.Hk);
  const int64_t i = blockIdx.x / a.Hq;
  const int64_t s = blockIdx.y;
  int64_t row, keys;
  int64_t last;  // last key seen
  if constexpr (CACHED) {
    int64_t q0 = a.b.q_start[s], q1 = a.b.q_start[s + 1];
    q0 = q0 < 0 ? 0 : q0 > a.T ? a.T : q0;
    q1 = q1 < q0 ? q0 : q1 > a.T ? a.T : q1;
    if (i >= q1 - q0) return;
    row = q0 + i;
    const int64_t len = a.b.kv_len[s];
    keys = len < a.max_kv ? len : a.max_kv;
    last = a.causal ? len - (q1 - q0) + i : keys - 1;
  } else {
    row = s * a.max_new + i;
    keys = a.max_kv;
    if (a.kv_len && a.kv_len[s] < keys) keys = a.kv_len[s];
    last = keys - 1;
  }
  if (last + 1 < keys) keys = last + 1;
  const uint16_t *q = CACHED ? a.q.p + row * a.q.ts + hq * a.q.hs : a.q.p + s * a.q.bs + i * a.q.ts + hq * a.q.hs;
  for (int d = lane; d < D; d += 64) qs[d] = __uint_as_float((uint32_t)q[d] << 16) * a.scale;
  __syncthreads();
  float m = -INFINITY, l = 0.0f, o[4] = {0, 0, 0, 0};
  auto page_of = [&](int64_t j) {
    int64_t p = a.b.pt[s * a.b.width + j / a.c.P];
    return (p < 0 ? 0 : p >= a.c.pages ? a.c.pages - 1 : p) * a.c.H + h;
  };
  for (int64_t j0 = 0; j0 < keys; j0 += 64) {
    const int64_t j = j0 + lane;
    float x = -INFINITY;
    bool seen = j < keys;
    if constexpr (!CACHED)
      if (seen && a.mask) seen = a.mask[s * a.mask_stride + j] != 0;
    if (seen) {
      x = 0.0f;
      if constexpr (CACHED) {
        const int64_t page = page_of(j);
        const int8_t *k = a.c.kc + (page * a.c.P + j % a.c.P) * D;
        for (int d = 0; d < D; ++d) x = __builtin_fmaf(qs[d], (float)k[d], x);
        x *= a.c.ks[page];
      } else {
        const uint16_t *k = a.k.p + s * a.k.bs + j * a.k.ts + h * a.k.hs;
        for (int d = 0; d < D; ++d) x = __builtin_fmaf(qs[d], __uint_as_float((uint32_t)k[d] << 16), x);
      }
    }
    float top = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
      const float y = __shfl_xor(top, d);
      top = y > top || y != y ? y : top;
    }
    if (top == -INFINITY) continue;  // the whole step is masked (uniform)
    const float to = top > m || top != top ? top : m;
    const float shrink = __expf(m - to);
    const float p = seen ? __expf(x - to) : 0.0f;
    float sum = p;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    l = l * shrink + sum;
    m = to;
    __syncthreads();
    ps[lane] = p;
    __syncthreads();
    const int n = (int)(keys - j0 < 64 ? keys - j0 : 64);
#pragma unroll
    for (int c = 0; c < 4; ++c) o[c] *= shrink;
    for (int t = 0; t < n; ++t) {
      const float w = ps[t];
      if constexpr (CACHED) {
        const int64_t page = page_of(j0 + t);
        const int off = (int)((j0 + t) % a.c.P);
        const float ws = w * a.c.vs[page];
        const int8_t *v = a.c.vc + page * a.c.P * D + (int64_t)(off / 16) * D * 16 + off % 16;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (lane + 64 * c < D) o[c] = __builtin_fmaf(ws, (float)v[(lane + 64 * c) * 16], o[c]);
      } else {
        if (a.mask && a.mask[s * a.mask_stride + j0 + t] == 0) continue;
        const uint16_t *v = a.v.p + s * a.v.bs + (j0 + t) * a.v.ts + h * a.v.hs;
#pragma unroll
        for (int c = 0; c < 4; ++c)
          if (lane + 64 * c < D) o[c] = __builtin_fmaf(w, __uint_as_float((uint32_t)v[lane + 64 * c] << 16), o[c]);
      }
    }
  }
  uint16_t *out = a.out + (row * a.Hq + hq) * D;
#pragma unroll
  for (int c = 0; c < 4; ++c)
    if (lane + 64 * c < D) out[lane + 64 * c] = (uint16_t)f32_to_bf16(l != 0.0f ? o[c] / l : 0.0f);
}

}  // namespace

size_t attention_workspace(bool, int64_t, int, int, int, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_attention(bool cached, const AttnArgs &a, void *, hipStream_t s) {
  const dim3 grid((unsigned)(a.max_new * a.Hq), (unsigned)a.seqs);
  if (cached)
    attention_row_kernel<true><<<grid, 64, 0, s>>>(a);
  else
    attention_row_kernel<false><<<grid, 64, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace fq
