// Attention over the 8-bit paged cache and over bf16 states: choice of kernel and split, and the
// join of split results.
#include "fq_attn_launch.hpp"

namespace fq {
namespace {

// Rows of one key head up to which the keys are streamed for 16 rows at a time.
constexpr int kStreamRows = 16;

struct Plan {
  bool stream;
  int64_t chunk;
  int splits;
};

// Workgroups of both kernels hold four waves and two of them fit a compute unit, so 512 fill the
// card.  Where the rows alone give fewer, or few rows leave ragged lengths to balance, the tokens
// are split.
Plan plan_attention(int Hq, int Hk, int64_t seqs, int64_t max_new, int64_t max_kv) {
  Plan p;
  const int64_t rows = max_new * (Hq / Hk);
  p.stream = rows <= kStreamRows;
  const int64_t per = p.stream ? 16 : attention_tile_rows();
  const int64_t groups = seqs * Hk * ((rows + per - 1) / per);
  const int64_t unit = p.stream ? 256 : 128;           // least tokens of a workgroup
  const int64_t want = p.stream ? 2048 : 512;          // workgroups
  int64_t splits = groups >= want ? 1 : want / groups;
  const int64_t most = (max_kv + unit - 1) / unit;
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  p.chunk = ((max_kv + splits - 1) / splits + unit - 1) / unit * unit;
  p.splits = p.chunk > 0 ? (int)((max_kv + p.chunk - 1) / p.chunk) : 1;
  if (p.splits <= 1) {
    p.splits = 1;
    p.chunk = (int64_t)1 << 40;
  }
  return p;
}

// One row a wave: the weighted mean of its parts.
template <bool CACHED>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a, Split sp) {
  const int lane = threadIdx.x % 64;
  const int D = a.D, G = a.Hq / a.Hk;
  const int64_t s = blockIdx.y;
  const int64_t per_seq = a.max_new * a.Hq;
  const int64_t x = (int64_t)blockIdx.x * 4 + threadIdx.x / 64;
  if (x >= per_seq) return;
  const Rows rows = sequence_queries<CACHED>(a, s);
  const int64_t i = x / a.Hq;
  const int hq = (int)(x - i * a.Hq), h = hq / G;
  if (i >= rows.n) return;
  const int64_t end = rows.end(i);
  const int parts = end <= 0 ? 0 : (int)((end + sp.chunk - 1) / sp.chunk);
  const int64_t stride = a.seqs * a.Hk * a.max_new * G;
  const int64_t at = (s * a.Hk + h) * (a.max_new * G) + i * G + hq % G;
  float m = -FLT_MAX;
  for (int p = lane; p < parts; p += 64) m = maxf(m, sp.ml[p * stride + at].x);
#pragma unroll
  for (int d = 1; d < 64; d *= 2) m = maxf(m, __shfl_xor(m, d));
  float o[4] = {0, 0, 0, 0}, l = 0.0f;
  if (4 * lane < D)
    for (int p = 0; p < parts; ++p) {
      const float2 ml = sp.ml[p * stride + at];
      const float w = exp2_fast(ml.x - m);
      const float4 v = *reinterpret_cast<const float4 *>(sp.o + (p * stride + at) * D + 4 * lane);
      l += ml.y * w;
      o[0] += v.x * w, o[1] += v.y * w, o[2] += v.z * w, o[3] += v.w * w;
    }
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  if (4 * lane < D)
    *reinterpret_cast<uint2 *>(a.out + ((rows.q0 + i) * a.Hq + hq) * D + 4 * lane) =
        make_uint2(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv));
}

}  // namespace

size_t attention_workspace(int Hq, int Hk, int D, int64_t seqs, int64_t max_new, int64_t max_kv) {
  const Plan p = plan_attention(Hq, Hk, seqs, max_new, max_kv);
  if (p.splits <= 1) return 0;
  return (size_t)p.splits * (size_t)seqs * (size_t)max_new * Hq * (D + 2) * 4;
}

hipError_t launch_attention(bool cached, const AttnArgs &a, void *ws, hipStream_t s) {
  const Plan p = plan_attention(a.Hq, a.Hk, a.seqs, a.max_new, a.max_kv);
  Split sp{p.chunk, p.splits, static_cast<float *>(ws), nullptr};
  if (p.splits > 1) sp.ml = reinterpret_cast<float2 *>(sp.o + (size_t)p.splits * a.seqs * a.max_new * a.Hq * a.D);
  hipError_t e = p.stream ? launch_attention_stream(cached, a, sp, s) : launch_attention_tile(cached, a, sp, s);
  if (e != hipSuccess || p.splits <= 1) return e;
  const dim3 grid((unsigned)((a.max_new * a.Hq + 3) / 4), (unsigned)a.seqs);
  if (cached)
    attention_join_kernel<true><<<grid, 256, 0, s>>>(a, sp);
  else
    attention_join_kernel<false><<<grid, 256, 0, s>>>(a, sp);
  return hipGetLastError();
}

}  // namespace fq
