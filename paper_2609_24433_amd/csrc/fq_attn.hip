// Attention over the 8-bit paged cache and over bf16 states: choice of kernel and split, and the
// join of split results.
#include "fq_attn_launch.hpp"

namespace fq {
namespace {

// Rows of one key head up to which the keys are streamed for 16 rows at a time, every 16 reading
// them again (from the caches).  8 sequences of up to 8192 tokens in the cache, 8 key heads of 128:
// 32 rows take 26 us (tiles 50), 48 rows 29 (49), 64 rows 42 (52).  8 samples of 4000 states, 16 heads
// of 128: 32 rows 95 us (tiles 96), 50 rows 141 (97).
constexpr int kStreamRowsCached = 64, kStreamRowsStates = 32;

// Streaming waves of 64 tokens up to which calls with more rows stream too: the card has a place for
// each, and a tile's walk would take longer than all of them (head above 128: half as many fit).  One
// sequence of 866 tokens, 8 query heads on one of 256: 50 rows of tokens, 350 waves, 14 us (tiles 20),
// 100, 700 waves, 21 (21); 4 key heads of 64, 200 rows each: 728 waves, 9.8 us (12.0).  50 queries
// against 816 states, 16 heads on 8 of 128: 728 waves, 11 us (17).
constexpr int kStreamWaves = 1024;

struct Plan {
  int rows;   // of a workgroup: 16 streaming, 128 or 256 with tiles
  int chunk;  // tokens of a part
  int splits;
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Streaming: parts of 64 KB of keys and values (256 cached tokens of head 128), so that waves of
// ragged sequences end evenly: 64 sequences of up to 8192 tokens, head 128, take 80 us, with 32 KB 85
// and with 128 KB 81; 32 of up to 4096, head 256, take 30, 33 and 37.  Parts get longer where there
// would be more than 32768 of them (their results cost room and time) and shorter, down to a tile,
// where there are too few to fill the card: one sequence of 877 tokens, head 256, takes 10 us with 64
// tokens a part, 19 with 128, 28 with 256.
// Tiles: 256 rows a workgroup of eight waves where there are more than 128 rows and the head size
// leaves the registers (head 128, 4096 rows over 8190 tokens: 422 us, with 128 rows 457), one a
// compute unit; of 128 rows two fit with heads of up to 128, one above (139 KB of LDS).  Tokens are
// split only to fill the card once, 128 or more a part: 8 query heads on one key head of 256, 816 tokens over 1632
// take 39 us, split for two workgroups a unit 50, 4096 over 4096 158 and 181; 1500 over 6000, head 160,
// 135 and 122, where 94 row tiles leave a quarter of the card idle.
Plan plan_attention(bool cached, int Hq, int Hk, int D, int64_t seqs, int64_t max_new, int64_t max_kv) {
  Plan p;
  const int64_t rows = max_new * (Hq / Hk);
  const double waves = (double)(seqs * Hk) * ceil_div(rows, 16) * ceil_div(max_kv, 64);
  const bool stream = rows <= (cached ? kStreamRowsCached : kStreamRowsStates) || waves <= (D > 128 ? kStreamWaves / 2 : kStreamWaves);
  p.rows = stream ? 16 : rows > 128 && D > 64 && D <= 128 ? 256 : 128;
  const int64_t groups = seqs * Hk * ceil_div(rows, p.rows);
  int64_t chunk;
  if (stream) {
    chunk = ceil_div(ceil_div(max_kv * groups, 32768), 64) * 64;
    const int64_t least = 65536 / ((cached ? 2 : 4) * D) / 64 * 64;
    if (chunk < least) chunk = least;
    while (chunk > 64 && groups * ceil_div(max_kv, chunk) < 1024) chunk = ceil_div(chunk / 2, 64) * 64;
  } else {
    const int64_t want = p.rows == 256 || D > 128 ? 256 : 512, splits = groups >= want ? 1 : want / groups;
    chunk = ceil_div(ceil_div(max_kv, splits), 128) * 128;
  }
  p.splits = max_kv > chunk ? (int)ceil_div(max_kv, chunk) : 1;
  p.chunk = p.splits > 1 ? (int)chunk : 1 << 30;
  return p;
}

// A row's result from its parts, 4 channels a lane: `lanes` lanes a part, `ways` parts of a row at
// once (each way keeps its own maximum).  A workgroup has 256 / (lanes ways)
// units; a unit is a row, or with fewer lanes than channels / 4 a slice of its channels.  Bound by the
// latency of its loads: 32 rows of 512 parts, head 128, 8.4 MB, 6.3 us, 0.2 of its waves' time vector work (the ways
// joined one after another through LDS: 10.7 us); 8 rows of 14 parts, 3.5 to 4.6 us, mostly launch.
template <bool CACHED>
__global__ __launch_bounds__(256) void attention_join_kernel(AttnArgs a, Split sp, int log_lanes, int log_ways, int slices) {
  __shared__ float4 os[256];
  __shared__ float2 mls[256];
  const int D = a.D, G = a.Hq / a.Hk;
  const int way = (threadIdx.x >> log_lanes) & ((1 << log_ways) - 1);
  const int64_t s = blockIdx.y;
  const int64_t unit = ((int64_t)blockIdx.x << (8 - log_lanes - log_ways)) + (threadIdx.x >> (log_lanes + log_ways));
  const int64_t x = unit / slices;
  const int c = (int)(unit - x * slices) << log_lanes | (threadIdx.x & ((1 << log_lanes) - 1));
  const Rows rows = sequence_queries<CACHED>(a, s);
  const int64_t i = x / a.Hq;
  const int hq = (int)(x - i * a.Hq), h = hq / G;
  const bool row = i < rows.n;
  const int end = row ? rows.end((int)i) : 0;
  const int parts = (int)(((int64_t)end + sp.chunk - 1) / sp.chunk);
  const int64_t stride = a.seqs * a.Hk * a.max_new * G;
  const int64_t at = (s * a.Hk + h) * (a.max_new * G) + i * G + hq % G;
  const bool in = 4 * c < D;
  float m = -FLT_MAX, l = 0.0f;
  float4 o = make_float4(0, 0, 0, 0);
  auto join = [&](float2 ml, float4 v) {
    const float to = maxf(m, ml.x), w0 = exp2_fast(m - to), w1 = exp2_fast(ml.x - to);
    m = to;
    l = l * w0 + ml.y * w1;
    o = make_float4(o.x * w0 + v.x * w1, o.y * w0 + v.y * w1, o.z * w0 + v.z * w1, o.w * w0 + v.w * w1);
  };
#pragma unroll 4
  for (int p = way; p < parts; p += 1 << log_ways)
    join(sp.ml[p * stride + at], in ? *reinterpret_cast<const float4 *>(sp.o + (p * stride + at) * D + 4 * c) : make_float4(0, 0, 0, 0));
  // the ways of a wave by exchange, then the waves of a unit through LDS
  for (int bit = log_lanes; bit < log_lanes + log_ways && bit < 6; ++bit) {
    const int with = 1 << bit;
    join(make_float2(__shfl_xor(m, with), __shfl_xor(l, with)),
         make_float4(__shfl_xor(o.x, with), __shfl_xor(o.y, with), __shfl_xor(o.z, with), __shfl_xor(o.w, with)));
  }
  if (log_lanes + log_ways > 6) {
    os[threadIdx.x] = o;
    mls[threadIdx.x] = make_float2(m, l);
    __syncthreads();
    if (way > 0) return;
    for (int w = 1; w < 1 << (log_lanes + log_ways - 6); ++w) join(mls[threadIdx.x + 64 * w], os[threadIdx.x + 64 * w]);
  }
  if (way > 0) return;
  if (!row || !in) return;
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  *reinterpret_cast<uint2 *>(a.out + ((rows.q0 + i) * a.Hq + hq) * D + 4 * c) =
      make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
}

}  // namespace

size_t attention_workspace(bool cached, int Hq, int Hk, int D, int64_t seqs, int64_t max_new, int64_t max_kv) {
  const Plan p = plan_attention(cached, Hq, Hk, D, seqs, max_new, max_kv);
  if (p.splits <= 1) return 0;
  return (size_t)p.splits * (size_t)seqs * (size_t)max_new * Hq * (D + 2) * 4;
}

hipError_t launch_attention(bool cached, const AttnArgs &a, void *ws, hipStream_t s) {
  const Plan p = plan_attention(cached, a.Hq, a.Hk, a.D, a.seqs, a.max_new, a.max_kv);
  Split sp{p.chunk, p.splits, static_cast<float *>(ws), nullptr};
  if (p.splits > 1) sp.ml = reinterpret_cast<float2 *>(sp.o + (size_t)p.splits * a.seqs * a.max_new * a.Hq * a.D);
  hipError_t e = p.rows == 16 ? launch_attention_stream(cached, a, sp, s) : launch_attention_tile(cached, a, sp, p.rows, s);
  if (e != hipSuccess || p.splits <= 1) return e;
  // channels over lanes, slices of 16 where whole rows would leave the card empty; then parts over ways
  int log_lanes = 2, log_ways = 0, slices = 1;
  while ((4 << log_lanes) < a.D) ++log_lanes;
  while (log_lanes > 2 && p.splits > 32 && a.seqs * a.max_new * a.Hq * slices < 512) --log_lanes, slices *= 2;
  while (log_lanes + log_ways < 8 && (4 << log_ways) < p.splits) ++log_ways;
  const int per = 8 - log_lanes - log_ways;
  const dim3 grid((unsigned)((a.max_new * a.Hq * slices + (1 << per) - 1) >> per), (unsigned)a.seqs);
  if (cached)
    attention_join_kernel<true><<<grid, 256, 0, s>>>(a, sp, log_lanes, log_ways, slices);
  else
    attention_join_kernel<false><<<grid, 256, 0, s>>>(a, sp, log_lanes, log_ways, slices);
  return hipGetLastError();
}

}  // namespace fq
