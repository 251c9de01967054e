// Attention for few query rows: up to 16 rows of one key head, where the keys and values are read
// once from memory.  A workgroup is one wave that walks its part of the tokens, a tile at a time
// straight from memory into the operands of the matrix instruction: waves share nothing, so a
// wave that ends makes room for the next at once, whatever the sequences' lengths.
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
__global__ __launch_bounds__(64, DP == 256 ? 2 : 3) void attention_stream_kernel(AttnArgs a, Split sp, int row_tiles) {
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
  const int lp = CACHED ? 31 - __builtin_clz(a.c.P) : 0;

  // row i of product t is token PER (i / 4) + 4 t + i % 4
  const int krow = PER * (col / 4) + col % 4;
  uint4 kr[NB][C][CACHED ? 1 : 2];
  uint4 vr[CACHED ? DT : DP / 16];
  int64_t page_k = -1, page_v = -1;  // of this lane's key rows and of its lane group's values, times heads
  float ks = 0.0f, vs = 0.0f;
  uint32_t bits = ~0u;

  auto find = [&](int j0) {
    if constexpr (CACHED) {
      const int jk = j0 + 16 * (col / 4), jv = j0 + 16 * g;
      page_k = jk < rows.keys ? cache_page(a, s, jk >> lp) * a.c.H + h : -1;
      page_v = jv < rows.keys ? cache_page(a, s, jv >> lp) * a.c.H + h : -1;
    } else {
      const int j = j0 + lane % 32;
      bool on = j < rows.keys;
      if (on && a.mask) on = a.mask[s * a.mask_stride + j] != 0;
      bits = (uint32_t)__ballot(on);
    }
  };
  auto fetch_keys = [&](int j0) {
    if constexpr (CACHED) {
      ks = page_v >= 0 ? a.c.ks[page_v] : 0.0f;
      vs = page_v >= 0 ? a.c.vs[page_v] : 0.0f;
      const int8_t *base = a.c.kc + (page_k * a.c.P + (int)((j0 + krow) & (a.c.P - 1))) * D;
#pragma unroll
      for (int t = 0; t < NB; ++t)
#pragma unroll
        for (int c = 0; c < C; ++c) {
          kr[t][c][0] = make_uint4(0, 0, 0, 0);
          if (page_k >= 0 && 64 * c + 16 * g < D)
            kr[t][c][0] = *reinterpret_cast<const uint4 *>(base + 4 * t * D + 64 * c + 16 * g);
        }
    } else {
      const uint16_t *base = a.k.p + s * a.k.bs + h * a.k.hs + (int64_t)(j0 + krow) * a.k.ts + 16 * g;
#pragma unroll
      for (int t = 0; t < NB; ++t) {
        const bool on = bits >> (krow + 4 * t) & 1;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            kr[t][c][e] = make_uint4(0, 0, 0, 0);
            if (on && 64 * c + 16 * g < D)
              kr[t][c][e] = *reinterpret_cast<const uint4 *>(base + 4 * t * a.k.ts + 64 * c + 8 * e);
          }
      }
    }
  };
  auto fetch_values = [&](int j0) {
    if constexpr (CACHED) {
      const int8_t *base = a.c.vc + page_v * a.c.P * D + (int64_t)((j0 + 16 * g) & (a.c.P - 1)) * D + col * 16;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        vr[i] = make_uint4(0, 0, 0, 0);
        if (page_v >= 0 && 16 * i < D) vr[i] = *reinterpret_cast<const uint4 *>(base + 256 * i);
      }
    } else {
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) {
        const int u = lane + 64 * i, token = u / (DP / 8), piece = u % (DP / 8);
        vr[i] = make_uint4(0, 0, 0, 0);
        if ((bits >> token & 1) && 8 * piece < D)
          vr[i] = *reinterpret_cast<const uint4 *>(a.v.p + s * a.v.bs + h * a.v.hs + (int64_t)(j0 + token) * a.v.ts + 8 * piece);
      }
    }
  };

  int j0 = c0;
  if (j0 < c1) {
    find(j0);
    fetch_keys(j0);
    fetch_values(j0);
  }
  for (; j0 < c1; j0 += NT) {
    const int next = j0 + NT;
    const uint32_t bits_now = bits;
    const float ks_now = ks, vs_now = vs;
    f32x4 st[NB];
#pragma unroll
    for (int t = 0; t < NB; ++t) {
      st[t] = f32x4{};
#pragma unroll
      for (int c = 0; c < C; ++c)
        if (64 * c < D)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint4 u;
            if constexpr (CACHED)
              u = e == 0 ? codes8_to_bf16(kr[t][c][0].x, kr[t][c][0].y) : codes8_to_bf16(kr[t][c][0].z, kr[t][c][0].w);
            else
              u = kr[t][c][e];
            st[t] = mfma16(__builtin_bit_cast(bf16x8, u), q[c][e], st[t]);
          }
    }
    if constexpr (!CACHED) {
#pragma unroll
      for (int i = 0; i < DP / 16; ++i) {
        const int u = lane + 64 * i, token = u / (DP / 8), piece = u % (DP / 8);
        *reinterpret_cast<uint4 *>(mine + token * kVStride + piece * 16) = vr[i];
      }
    }
    if (next < c1) {
      find(next);
      fetch_keys(next);
    }
    const float c = CACHED ? c_all * ks_now : c_all;
    const bool masked = j0 + NT > end_min || (!CACHED && bits_now != ~0u);
    uint32_t on = (1u << PER) - 1;
    if (masked) {
      const int left = end - (j0 + PER * g);
      on = left >= PER ? on : left <= 0 ? 0u : (1u << left) - 1;
      if (!CACHED) on &= bits_now >> (PER * g);
    }
    float x = -FLT_MAX;
#pragma unroll
    for (int t = 0; t < NB; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) x = maxf(x, !masked || (on >> (4 * t + e) & 1) ? st[t][e] : -FLT_MAX);
    float top = on ? maxf(x * c, -FLT_MAX) : -FLT_MAX;
    top = across16(across32(top, maxf), maxf);
    if (__any(top > m + 8.0f)) {
      const float to = maxf(m, top), shrink = exp2_fast(m - to);
      m = to;
      l *= shrink;
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= shrink;
    }
    bf16x8 p[NB / 2];
#pragma unroll
    for (int b = 0; b < NB / 2; ++b) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const bool seen = !masked || (on >> (8 * b + e) & 1);
        float y = exp2_fast(__builtin_fmaf(st[2 * b + e / 4][e % 4], c, -m));
        y = seen ? y : 0.0f;
        l += y;
        w[e] = CACHED ? (seen ? y * vs_now : 0.0f) : y;
      }
      p[b] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]),
                                                  pack_bf16(w[6], w[7])));
    }
    if constexpr (!CACHED) wave_lds_fence();
#pragma unroll
    for (int i = 0; i < DT; ++i)
      if (16 * i < D) {
        if constexpr (CACHED) {
          o[i] = mfma16(__builtin_bit_cast(bf16x8, codes8_to_bf16(vr[i].x, vr[i].y)), p[0], o[i]);
          o[i] = mfma16(__builtin_bit_cast(bf16x8, codes8_to_bf16(vr[i].z, vr[i].w)), p[1], o[i]);
        } else {
          const uint8_t *at = mine + (8 * g + col / 4) * kVStride + (16 * i + 4 * (col % 4)) * 2;
          const uint2 x0 = lds_read_transposed(at), x1 = lds_read_transposed(at + 4 * kVStride);
          o[i] = mfma16(__builtin_bit_cast(bf16x8, make_uint4(x0.x, x0.y, x1.x, x1.y)), p[0], o[i]);
        }
      }
    if constexpr (!CACHED) wave_lds_fence();
    if (next < c1) fetch_values(next);
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
