// Attention for few query rows: up to 16 rows of one key head, where the keys and values are read
// once from memory.  A workgroup is one wave that walks its part of the tokens, a tile at a time
// straight from memory into the operands of the matrix instruction: waves share nothing, so a
// wave that ends makes room for the next at once, whatever the sequences' lengths.
//
// Per row, with scores s_j in log2 units and m a running bound on them: l = sum 2^(s_j - m) and
// o = sum 2^(s_j - m) v_j, both rescaled when m moves; the result is o / l.  Parts of a long context
// leave (m, l, o) for the join.
//
// Bound by memory where there are many sequences (the first case below moves 351 MB at 4.8 TB/s in this
// kernel, the second 147 at 5.6, by the counters), by the latency of a wave's walk and of the join's
// launch where there are few.  Measured, with the join: 64 sequences of up to 8192 tokens in the
// cache, 8 key heads of 128, 32 query heads: 80 us, 4.1 TB/s; two of 131071 tokens, 2 key heads, 33 us,
// 4.0 TB/s; one of 877 tokens, one key head of 256, 10 us, and 50 tokens of one of 866 14 us; a query in
// each of 24 samples of up to 1500 bf16 states, 16 heads of 128: 38 us, 4.3 TB/s.
#include "fq_attn_device.hpp"
#include "fq_attn_launch.hpp"

namespace fq {
namespace {

// Tokens a wave takes at once.  A lane (row l % 16, group g = l / 16 of the operands' k) holds the
// scores of NT / 4 consecutive tokens, 16 g .. of 64 or 8 g .. of 32: cached tiles have 64, one
// 16-token group of the cache a lane group; states 32, of twice the bytes.
template <bool CACHED>
struct Tile {
  static constexpr int kTokens = CACHED ? 64 : 32;
  static constexpr int kBlocks = kTokens / 16;  // 16-token products
};

template <bool CACHED, int DP>
__global__ __launch_bounds__(64, DP == 256 ? 1 : 2) void attention_stream_kernel(AttnArgs a, Split sp, int row_tiles) {
  constexpr int NT = Tile<CACHED>::kTokens, NB = Tile<CACHED>::kBlocks, PER = NT / 4;
  constexpr int C = DP / 64;  // 64-channel steps: a lane group reads 16 channels of each
  constexpr int DT = DP / 16;
  constexpr int kVStride = 2 * DP + 32;  // values of the wave's tile in LDS (states): bytes of a token
  __shared__ __align__(16) uint8_t mine[CACHED ? 16 : 32 * kVStride];
  const int lane = threadIdx.x;
  const int col = lane % 16, g = lane / 16;
  const int D = a.D, G = a.Hq / a.Hk;
  const int h = blockIdx.x % a.Hk;
  const int tile_row = blockIdx.x / a.Hk % row_tiles;
  const int part = blockIdx.x / a.Hk / row_tiles;
  const int64_t s = blockIdx.y;
  const Rows rows = sequence_queries<CACHED>(a, s);
  const int total = rows.n * G, r0 = tile_row * 16;
  if (r0 >= total) return;
  const int last_row = total - r0 > 16 ? r0 + 15 : total - 1;
  const int c0 = part * sp.chunk;
  const int end_max = rows.end(last_row / G), end_min = rows.end(r0 / G);
  const int c1 = end_max - c0 > sp.chunk ? c0 + sp.chunk : end_max;
  if (c1 <= c0 && part > 0) return;  // no row of it has a partial result here

  const int r = r0 + col;
  const bool live = r < total;
  const int qi = live ? r / G : 0;
  const int hq = h * G + (live ? r - qi * G : 0);
  const int end = live ? rows.end(qi) : 0;

  // channel order of the first product: step (c, e) has channels 64 c + 16 g + 8 e ..
  bf16x8 q[C][2];
  {
    const uint16_t *p = CACHED ? a.q.p + (rows.q0 + qi) * a.q.ts + hq * a.q.hs : a.q.p + s * a.q.bs + qi * a.q.ts + hq * a.q.hs;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        uint4 u = make_uint4(0, 0, 0, 0);
        if (live && 64 * c + 16 * g < D) u = *reinterpret_cast<const uint4 *>(p + 64 * c + 16 * g + 8 * e);
        q[c][e] = __builtin_bit_cast(bf16x8, u);
      }
  }
  f32x4 o[DT];
#pragma unroll
  for (int i = 0; i < DT; ++i) o[i] = f32x4{};
  float m = -FLT_MAX, l = 0.0f;
  const float c_all = a.scale * 1.4426950408889634f;
  const int last_key = rows.keys - 1;

  // Loads are unconditional, at addresses that are there: channels from D on meet zeros of q or go
  // to channels nobody reads, tokens past the last one have weights of zero.
  // row i of product t is token PER (i / 4) + 4 t + i % 4
  const int krow = PER * (col / 4) + col % 4;
  struct Loaded {
    uint4 k[NB][C][CACHED ? 1 : 2];
    uint4 v[CACHED ? DT : DP / 16];
    float ks, vs;
    uint32_t bits;  // states: seen places
  };
  // One tile, refilled as its halves are used up: the keys' loads run under the softmax and the
  // second product, the values' under the next tile's first.  (A second tile of registers measured
  // no better: decode of 64 sequences 90 us for 81.)
  Loaded now;
  uint32_t on_next = 0;  // states: whether place lane % 32 of the tile to come is seen
  // cache: pages of the groups of this lane's key rows and of its values, looked up a tile ahead
  const int lp = CACHED ? 31 - __builtin_clz(a.c.P) : 0, in_page = a.c.P - 1;
  const int32_t *pt = CACHED ? a.b.pt + s * a.b.width : nullptr;
  int page_k = 0, page_v = 0;
  int64_t at_k = 0, at_v = 0;
  auto look_up = [&](int j0) {
    if constexpr (CACHED) {
      const int jk = j0 + 16 * (col / 4), jv = j0 + 16 * g;
      page_k = pt[(jk < last_key ? jk : last_key) >> lp];
      page_v = pt[(jv < last_key ? jv : last_key) >> lp];
    } else {
      const int j = j0 + lane % 32;
      on_next = j <= last_key;
      if (a.mask) on_next &= a.mask[s * a.mask_stride + (j <= last_key ? j : last_key)] != 0;
    }
  };
  auto fetch_keys = [&](int j0) {
    if constexpr (CACHED) {
      at_k = (int64_t)clamp_page(page_k, a.c.pages) * a.c.H + h;
      at_v = (int64_t)clamp_page(page_v, a.c.pages) * a.c.H + h;
      now.ks = a.c.ks[at_v];
      now.vs = a.c.vs[at_v];
      const int8_t *base = a.c.kc + (at_k * a.c.P + ((j0 + krow) & in_page)) * D;
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int c = 0; c < C; ++c)
          now.k[t][c][0] = *reinterpret_cast<const uint4 *>(base + (4 * t * D + (64 * c + 16 * g < D ? 64 * c + 16 * g : 0)));
    } else {
      now.bits = (uint32_t)__ballot(on_next != 0);
      const uint16_t *base = a.k.p + s * a.k.bs + h * a.k.hs;
#pragma unroll
      for (int t = 0; t < NB; ++t) {
        const int j = j0 + krow + 4 * t;
        const uint16_t *row = base + (int64_t)(j < last_key ? j : last_key) * a.k.ts;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            now.k[t][c][e] = *reinterpret_cast<const uint4 *>(row + (64 * c + 16 * g < D ? 64 * c + 16 * g + 8 * e : 0));
      }
    }
  };
  auto fetch_values = [&](int j0) {
    if constexpr (CACHED) {
      const int8_t *base = a.c.vc + (at_v * a.c.P + ((j0 + 16 * g) & in_page)) * D + col * 16;
#pragma unroll
      for (int i = 0; i < DT; ++i) now.v[i] = *reinterpret_cast<const uint4 *>(base + (16 * i < D ? 256 * i : 0));
    } else {
      const uint16_t *base = a.v.p + s * a.v.bs + h * a.v.hs;
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) {
        const int u = lane + 64 * i, j = j0 + u / (DP / 8), piece = 8 * (u % (DP / 8));
        now.v[i] = *reinterpret_cast<const uint4 *>(base + (int64_t)(j < last_key ? j : last_key) * a.v.ts + (piece < D ? piece : 0));
      }
    }
  };

  if (c0 < c1) {
    look_up(c0);
    fetch_keys(c0);
    fetch_values(c0);
    if (c0 + NT < c1) look_up(c0 + NT);
  }
  for (int j0 = c0; j0 < c1; j0 += NT) {
    const int next = j0 + NT;
    float c = CACHED ? c_all * now.ks : c_all;
    float v = CACHED ? now.vs : 1.0f;
    const uint32_t bits = CACHED ? ~0u : now.bits;
    f32x4 st[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t) st[t] = f32x4{};
#pragma unroll
    for (int i = 0; i < C; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int t = 0; t < NB; ++t) {
          uint4 u;
          if constexpr (CACHED)
            u = e == 0 ? codes8_to_bf16(now.k[t][i][0].x, now.k[t][i][0].y) : codes8_to_bf16(now.k[t][i][0].z, now.k[t][i][0].w);
          else
            u = now.k[t][i][e];
          if (!CACHED && D < DP && 64 * i + 16 * g >= D) u = make_uint4(0, 0, 0, 0);
          st[t] = mfma16(__builtin_bit_cast(bf16x8, u), q[i][e], st[t]);
        }
    if constexpr (!CACHED) {
      if (bits != ~0u)  // what unseen places hold must not reach the product
#pragma unroll
        for (int i = 0; i < DP / 16; ++i)
          if (!(bits >> ((lane + 64 * i) / (DP / 8)) & 1)) now.v[i] = make_uint4(0, 0, 0, 0);
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) {
        const int u = lane + 64 * i, token = u / (DP / 8), piece = u % (DP / 8);
        *reinterpret_cast<uint4 *>(mine + token * kVStride + piece * 16) = now.v[i];
      }
    }
    if (next < c1) fetch_keys(next);
    // Unseen places' scores become -infinity, with the scale applied here, so that a scale that is 0
    // or NaN reaches only what is seen; a NaN scale of the values goes by the scores.
    if (j0 + NT > end_min || (!CACHED && bits != ~0u)) {
      const int left = end - (j0 + PER * g);
      uint32_t on = left >= PER ? (1u << PER) - 1 : left <= 0 ? 0u : (1u << left) - 1;
      if (!CACHED) on &= bits >> (PER * g);
      const float bad = CACHED ? v - v : 0.0f;
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) st[t][e] = (on >> (4 * t + e) & 1) ? __builtin_fmaf(st[t][e], c, bad) : -INFINITY;
      c = 1.0f;
      if (CACHED && bad != 0.0f) v = 1.0f;
    }
    float x = st[0][0];
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) x = maxf(x, st[t][e]);
    const float top = x * c;
    // the running maximum moves only where it has to: a weight up to 2^8 is as exact as one up to 1
    if (__any(top > m + 8.0f)) {
      const float to = maxf(m, across16(across32(maxf(top, -FLT_MAX), maxf), maxf)), shrink = exp2_fast(m - to);
      m = to;
      l *= shrink;
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] *= shrink;
    }
    // Weights enter the product as two bf16 values each, 16 bits of them: the matrix unit has the time
    // while the keys and values come from memory.  (With one, the result's error against 64 bits is
    // 0.0024 of its size for 0.0016, bf16's own, and the times are the same within 2 %.)  Values of states may
    // be infinite: their weights are cut off, not rounded, and the second value is at least 2^-24 of the weight, so
    // that neither meets an infinity with another sign or as 0 (15 bits).  A cache's codes are finite.
    uint4 p[NB / 2], rest[NB / 2];
#pragma unroll
    for (int b = 0; b < NB / 2; ++b) {
      uint32_t w[4], r[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float w0 = exp2_fast(__builtin_fmaf(st[2 * b + e / 2][2 * (e % 2)], c, -m));
        float w1 = exp2_fast(__builtin_fmaf(st[2 * b + e / 2][2 * (e % 2) + 1], c, -m));
        l += w0;
        l += w1;
        if constexpr (CACHED) {
          w0 *= v, w1 *= v;
          w[e] = pack_bf16(w0, w1);
          r[e] = pack_bf16(w0 - bf16_lo(w[e]), w1 - bf16_hi(w[e]));
        } else {
          w[e] = __builtin_amdgcn_perm(__float_as_uint(w1), __float_as_uint(w0), 0x07060302u);
          r[e] = pack_bf16(__builtin_fmaf(w0, 0x1p-24f, w0 - bf16_lo(w[e])), __builtin_fmaf(w1, 0x1p-24f, w1 - bf16_hi(w[e])));
        }
      }
      p[b] = make_uint4(w[0], w[1], w[2], w[3]);
      rest[b] = make_uint4(r[0], r[1], r[2], r[3]);
    }
    auto weigh = [&](int i, uint4 x, int b) {
      o[i] = mfma16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, p[b]), o[i]);
      o[i] = mfma16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, rest[b]), o[i]);
    };
    if constexpr (!CACHED) wave_lds_fence();
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      if constexpr (CACHED) {
        weigh(i, codes8_to_bf16(now.v[i].x, now.v[i].y), 0);
        weigh(i, codes8_to_bf16(now.v[i].z, now.v[i].w), 1);
      } else {
        const uint8_t *at = mine + (8 * g + col / 4) * kVStride + (16 * i + 4 * (col % 4)) * 2;
        const uint2 x0 = lds_read_transposed(at), x1 = lds_read_transposed(at + 4 * kVStride);
        weigh(i, make_uint4(x0.x, x0.y, x1.x, x1.y), 0);
      }
    }
    if constexpr (!CACHED) wave_lds_fence();
    if (next < c1) {
      fetch_values(next);
      if (next + NT < c1) look_up(next + NT);
    }
  }
  l = across16(across32(l, [](float x, float y) { return x + y; }), [](float x, float y) { return x + y; });
  if (!live) return;
  // a lane holds channels 16 i + 4 g .. of its row
  if (sp.splits > 1) {
    const int64_t at = (((int64_t)part * a.seqs + s) * a.Hk + h) * (a.max_new * G) + r;
    if (g == 0) sp.ml[at] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < DT; ++i)
      if (16 * i < D)
        *reinterpret_cast<float4 *>(sp.o + at * D + 16 * i + 4 * g) = make_float4(o[i][0], o[i][1], o[i][2], o[i][3]);
    return;
  }
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  uint16_t *out = a.out + ((rows.q0 + qi) * a.Hq + hq) * D;
#pragma unroll
  for (int i = 0; i < DT; ++i)
    if (16 * i < D)
      *reinterpret_cast<uint2 *>(out + 16 * i + 4 * g) =
          make_uint2(pack_bf16(o[i][0] * inv, o[i][1] * inv), pack_bf16(o[i][2] * inv, o[i][3] * inv));
}

template <bool CACHED, int DP>
hipError_t launch(const AttnArgs &a, const Split &sp, hipStream_t s) {
  const int64_t row_tiles = (a.max_new * (a.Hq / a.Hk) + 15) / 16;
  attention_stream_kernel<CACHED, DP><<<dim3((unsigned)(a.Hk * row_tiles * sp.splits), (unsigned)a.seqs), 64, 0, s>>>(
      a, sp, (int)row_tiles);
  return hipGetLastError();
}

template <bool CACHED>
hipError_t launch_size(const AttnArgs &a, const Split &sp, hipStream_t s) {
  if (a.D <= 64) return launch<CACHED, 64>(a, sp, s);
  if (a.D <= 128) return launch<CACHED, 128>(a, sp, s);
  return launch<CACHED, 256>(a, sp, s);
}

}  // namespace

hipError_t launch_attention_stream(bool cached, const AttnArgs &a, const Split &sp, hipStream_t s) {
  return cached ? launch_size<true>(a, sp, s) : launch_size<false>(a, sp, s);
}

}  // namespace fq
