// Attention for many query rows: a workgroup of four waves holds 128 rows of one key head (32 a
// wave) and walks the keys in tiles of 64 that all four waves read from LDS.
#include "fq_attn_device.hpp"
#include "fq_attn_launch.hpp"

namespace fq {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 32 * kWaves, kTile = 64;

// LDS of a tile: keys [64][DP] bf16, the 16-byte pieces of a token's row swizzled; values
// transposed [DP][64 + 8] (cache) or [64][DP + 16] (states, read with the transposing read).
template <bool CACHED, int DP>
struct Lds {
  static constexpr int kKeys = kTile * DP * 2;
  static constexpr int kVStride = CACHED ? 2 * kTile + 16 : 2 * DP + 32;  // bytes of a row
  static constexpr int kValues = (CACHED ? DP : kTile) * kVStride;
  static constexpr int kBuffer = kKeys + kValues;
};
// Eight lanes that read one piece of tokens 0-3 and 16-19 (+ 4 a) meet eight bank groups.
__device__ __forceinline__ int swizzle(int token) { return (token & 3) | ((token >> 2) & 4); }

template <bool CACHED, int DP>
__global__ __launch_bounds__(kThreads, DP == 256 ? 1 : 2) void attention_tile_kernel(AttnArgs a, Split sp, int row_tiles) {
  extern __shared__ __align__(16) uint8_t lds[];
  using L = Lds<CACHED, DP>;
  constexpr int KU = kTile * (DP / 16) / kThreads;  // 16-channel pieces of keys a thread stages
  constexpr int VU = CACHED ? 4 * DP / kThreads : kTile * (DP / 8) / kThreads;
  const int tid = threadIdx.x, lane = tid % 64, wave = __builtin_amdgcn_readfirstlane(tid / 64);
  const int col = lane % 32, half = lane / 32;
  const int D = a.D, G = a.Hq / a.Hk;
  const int h = blockIdx.x % a.Hk;
  const int part = blockIdx.x / a.Hk % sp.splits;
  const int tile_row = row_tiles - 1 - blockIdx.x / a.Hk / sp.splits;  // longest rows first
  const int64_t s = blockIdx.y;
  const Rows rows = sequence_queries<CACHED>(a, s);
  const int64_t total = rows.n * G, r0 = (int64_t)tile_row * kRows;
  if (r0 >= total) return;

  // keys of the workgroup: its range, up to what its last row sees
  const int64_t last_row = r0 + kRows < total ? r0 + kRows - 1 : total - 1;
  const int64_t c0 = (int64_t)part * sp.chunk;
  int64_t c1 = rows.end(last_row / G);
  if (c1 > c0 + sp.chunk) c1 = c0 + sp.chunk;
  if (c1 <= c0 && part > 0) return;  // no row of it has a partial result here
  const int tiles = c1 > c0 ? (int)((c1 - c0 + kTile - 1) / kTile) : 0;

  // this lane's row, as the column of both products
  const int64_t r = r0 + wave * 32 + col;
  const bool live = r < total;
  const int64_t qi = live ? r / G : 0;
  const int hq = h * G + (int)(live ? r - qi * G : 0);
  const int64_t end = live ? rows.end(qi) : 0;
  bf16x8 q[DP / 16];
  {
    const uint16_t *p = CACHED ? a.q.p + (rows.q0 + qi) * a.q.ts + hq * a.q.hs : a.q.p + s * a.q.bs + qi * a.q.ts + hq * a.q.hs;
#pragma unroll
    for (int i = 0; i < DP / 16; ++i) {
      uint4 u = make_uint4(0, 0, 0, 0);
      if (live && 16 * i < D) u = *reinterpret_cast<const uint4 *>(p + 16 * i + 8 * half);
      q[i] = __builtin_bit_cast(bf16x8, u);
    }
  }
  // least and most that a row of the wave sees, for the masks
  const int64_t wr0 = r0 + wave * 32, wr1 = wr0 + 31 < total ? wr0 + 31 : total - 1;
  const int64_t end_min = wr0 < total ? rows.end(wr0 / G) : 0, end_max = wr0 < total ? rows.end(wr1 / G) : 0;

  f32x16 o[DP / 32];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) o[i] = f32x16{};
  float m = -FLT_MAX, l = 0.0f;
  const float c_all = a.scale * 1.4426950408889634f;

  // staging registers of the next tile
  uint4 kr[CACHED ? KU : 2 * KU], vr[VU];
  float ks[2], vs[2];
  uint64_t seen_bits = ~0ull;

  auto fetch = [&](int t) {
    const int64_t j0 = c0 + (int64_t)t * kTile;
    if constexpr (CACHED) {
      const int64_t hb = (int64_t)h;
      const int lp = 31 - __builtin_clz(a.c.P);
      // the 16-token group of a unit is the same for a whole wave
      auto group_page = [&](int g) -> int64_t {
        const int64_t j = j0 + 16 * g;
        return j < rows.keys ? cache_page(a, s, j >> lp) * a.c.H + hb : -1;
      };
#pragma unroll
      for (int i = 0; i < KU; ++i) {
        const int u = tid + i * kThreads, token = u / (DP / 16), piece = u % (DP / 16);
        const int64_t pg = group_page(__builtin_amdgcn_readfirstlane(token / 16));
        kr[i] = make_uint4(0, 0, 0, 0);
        if (pg >= 0 && 16 * piece < D)
          kr[i] = *reinterpret_cast<const uint4 *>(a.c.kc + (pg * a.c.P + (int)((j0 + token) & (a.c.P - 1))) * D + 16 * piece);
      }
#pragma unroll
      for (int i = 0; i < VU; ++i) {
        const int u = tid + i * kThreads, d = u % DP;
        const int g = __builtin_amdgcn_readfirstlane(u / DP);
        const int64_t pg = group_page(g);
        vr[i] = make_uint4(0, 0, 0, 0);
        if (pg >= 0 && d < D)
          vr[i] = *reinterpret_cast<const uint4 *>(a.c.vc + pg * a.c.P * D + ((int64_t)((j0 + 16 * g) & (a.c.P - 1)) * D + d * 16));
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int64_t pg = group_page(2 * i + half);
        ks[i] = pg >= 0 ? a.c.ks[pg] : 0.0f;
        vs[i] = pg >= 0 ? a.c.vs[pg] : 0.0f;
      }
    } else {
      const int64_t j = j0 + lane;
      bool on = j < rows.keys;
      if (on && a.mask) on = a.mask[s * a.mask_stride + j] != 0;
      seen_bits = __ballot(on);
#pragma unroll
      for (int i = 0; i < 2 * KU; ++i) {
        const int u = tid + i * kThreads, token = u / (DP / 8), piece = u % (DP / 8);
        kr[i] = make_uint4(0, 0, 0, 0);
        if ((seen_bits >> token & 1) && 8 * piece < D)
          kr[i] = *reinterpret_cast<const uint4 *>(a.k.p + s * a.k.bs + (j0 + token) * a.k.ts + h * a.k.hs + 8 * piece);
        vr[i] = make_uint4(0, 0, 0, 0);
        if ((seen_bits >> token & 1) && 8 * piece < D)
          vr[i] = *reinterpret_cast<const uint4 *>(a.v.p + s * a.v.bs + (j0 + token) * a.v.ts + h * a.v.hs + 8 * piece);
      }
    }
  };
  auto stage = [&](uint8_t *buf) {
    uint8_t *kb = buf, *vb = buf + L::kKeys;
    if constexpr (CACHED) {
#pragma unroll
      for (int i = 0; i < KU; ++i) {
        const int u = tid + i * kThreads, token = u / (DP / 16), piece = 2 * (u % (DP / 16)), sw = swizzle(token);
        *reinterpret_cast<uint4 *>(kb + token * DP * 2 + ((piece ^ sw) * 16)) = codes8_to_bf16(kr[i].x, kr[i].y);
        *reinterpret_cast<uint4 *>(kb + token * DP * 2 + (((piece + 1) ^ sw) * 16)) = codes8_to_bf16(kr[i].z, kr[i].w);
      }
#pragma unroll
      for (int i = 0; i < VU; ++i) {
        const int u = tid + i * kThreads, d = u % DP, g = u / DP;
        uint4 *to = reinterpret_cast<uint4 *>(vb + d * L::kVStride + g * 32);
        to[0] = codes8_to_bf16(vr[i].x, vr[i].y);
        to[1] = codes8_to_bf16(vr[i].z, vr[i].w);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 2 * KU; ++i) {
        const int u = tid + i * kThreads, token = u / (DP / 8), piece = u % (DP / 8);
        *reinterpret_cast<uint4 *>(kb + token * DP * 2 + ((piece ^ swizzle(token)) * 16)) = kr[i];
        *reinterpret_cast<uint4 *>(vb + token * L::kVStride + piece * 16) = vr[i];
      }
    }
  };

  float ks_now[2], vs_now[2];
  uint64_t bits = ~0ull;
  if (tiles > 0) {
    fetch(0);
    stage(lds);
    bits = seen_bits;
#pragma unroll
    for (int i = 0; i < 2; ++i) ks_now[i] = ks[i], vs_now[i] = vs[i];
  }
  for (int t = 0; t < tiles; ++t) {
    const uint8_t *kb = lds + (t & 1) * L::kBuffer, *vb = kb + L::kKeys;
    __syncthreads();
    if (t + 1 < tiles) fetch(t + 1);
    const int64_t j0 = c0 + (int64_t)t * kTile;
    if (j0 < end_max) {
      // S^T: row i = 8 x + 4 y + z of a 32-token block is token 16 y + 4 x + z
      const int token = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3);
      f32x16 st[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        st[b] = f32x16{};
        const uint8_t *row = kb + (32 * b + token) * DP * 2;
        const int sw = swizzle(token);
#pragma unroll
        for (int i = 0; i < DP / 16; ++i)
          if (16 * i < D) {
            const uint4 u = *reinterpret_cast<const uint4 *>(row + (((2 * i + half) ^ sw) * 16));
            st[b] = mfma32(__builtin_bit_cast(bf16x8, u), q[i], st[b]);
          }
      }
      float c[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) c[b] = CACHED ? c_all * ks_now[b] : c_all;
      // unseen places: beyond a row's end, or masked
      const bool masked = j0 + kTile > end_min || (!CACHED && bits != ~0ull);
      uint32_t on[2] = {0xFFFFu, 0xFFFFu};
      if (masked) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int64_t left = end - (j0 + 32 * b + 16 * half);
          on[b] = left >= 16 ? 0xFFFFu : left <= 0 ? 0u : (1u << left) - 1;
          if (!CACHED) on[b] &= (uint32_t)(bits >> (32 * b + 16 * half));
        }
      }
      float top = -FLT_MAX;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float x = -FLT_MAX;
        if (masked) {
#pragma unroll
          for (int e = 0; e < 16; ++e) x = maxf(x, (on[b] >> e & 1) ? st[b][e] : -FLT_MAX);
          if (on[b]) top = maxf(top, x * c[b]);
        } else {
#pragma unroll
          for (int e = 0; e < 16; ++e) x = maxf(x, st[b][e]);
          top = maxf(top, x * c[b]);
        }
      }
      top = across32(top, maxf);
      // the running maximum moves only where it has to: up to 2^8 above it a weight is as exact
      if (__any(top > m + 8.0f)) {
        const float to = maxf(m, top), shrink = exp2_fast(m - to);
        m = to;
        l *= shrink;
#pragma unroll
        for (int i = 0; i < DP / 32; ++i)
          if (32 * i < D) o[i] *= shrink;
      }
      bf16x8 p[2][2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float x = exp2_fast(__builtin_fmaf(st[b][e], c[b], -m));
          if (masked) x = (on[b] >> e & 1) ? x : 0.0f;
          l += x;
          w[e] = CACHED ? x * vs_now[b] : x;
          if (CACHED && masked) w[e] = (on[b] >> e & 1) ? w[e] : 0.0f;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e)
          p[b][e] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16(w[8 * e], w[8 * e + 1]), pack_bf16(w[8 * e + 2], w[8 * e + 3]),
                                                         pack_bf16(w[8 * e + 4], w[8 * e + 5]), pack_bf16(w[8 * e + 6], w[8 * e + 7])));
      }
      // O^T: a lane's weights 8 e .. 8 e + 7 are tokens 32 b + 16 half + 8 e ..
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
        if (32 * i < D) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              uint4 u;
              if constexpr (CACHED) {
                u = *reinterpret_cast<const uint4 *>(vb + (32 * i + col) * L::kVStride + (32 * b + 16 * half + 8 * e) * 2);
              } else {
                const int piece = lane % 16;
                const uint8_t *at = vb + (32 * b + 16 * half + 8 * e + piece / 4) * L::kVStride +
                                    (32 * i + 16 * ((lane >> 4) & 1) + 4 * (piece % 4)) * 2;
                const uint2 x = lds_read_transposed(at), y = lds_read_transposed(at + 4 * L::kVStride);
                u = make_uint4(x.x, x.y, y.x, y.y);
              }
              o[i] = mfma32(__builtin_bit_cast(bf16x8, u), p[b][e], o[i]);
            }
        }
    }
    if (t + 1 < tiles) {
      stage(lds + ((t + 1) & 1) * L::kBuffer);
      bits = seen_bits;
#pragma unroll
      for (int i = 0; i < 2; ++i) ks_now[i] = ks[i], vs_now[i] = vs[i];
    }
  }
  l = across32(l, [](float x, float y) { return x + y; });
  if (!live) return;
  // a lane holds channels 32 i + 8 x + 4 half + z of its row
  if (sp.splits > 1) {
    const int64_t at = ((part * a.seqs + s) * a.Hk + h) * (a.max_new * G) + r;
    if (half == 0) sp.ml[at] = make_float2(m, l);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int d = 32 * i + 8 * x + 4 * half;
        if (d < D)
          *reinterpret_cast<float4 *>(sp.o + at * D + d) = make_float4(o[i][4 * x], o[i][4 * x + 1], o[i][4 * x + 2], o[i][4 * x + 3]);
      }
    return;
  }
  const float inv = l != 0.0f ? 1.0f / l : 0.0f;
  uint16_t *out = a.out + ((rows.q0 + qi) * a.Hq + hq) * D;
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int d = 32 * i + 8 * x + 4 * half;
      if (d < D)
        *reinterpret_cast<uint2 *>(out + d) = make_uint2(pack_bf16(o[i][4 * x] * inv, o[i][4 * x + 1] * inv),
                                                        pack_bf16(o[i][4 * x + 2] * inv, o[i][4 * x + 3] * inv));
    }
}

template <bool CACHED, int DP>
hipError_t launch(const AttnArgs &a, const Split &sp, hipStream_t s) {
  static std::atomic<uint64_t> raised{0};
  const size_t lds = 2 * (size_t)Lds<CACHED, DP>::kBuffer;
  hipError_t e = allow_dynamic_lds(attention_tile_kernel<CACHED, DP>, lds, raised);
  if (e != hipSuccess) return e;
  const int64_t row_tiles = (a.max_new * (a.Hq / a.Hk) + kRows - 1) / kRows;
  attention_tile_kernel<CACHED, DP><<<dim3((unsigned)(a.Hk * row_tiles * sp.splits), (unsigned)a.seqs), kThreads, lds, s>>>(
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

int attention_tile_rows() { return kRows; }

hipError_t launch_attention_tile(bool cached, const AttnArgs &a, const Split &sp, hipStream_t s) {
  return cached ? launch_size<true>(a, sp, s) : launch_size<false>(a, sp, s);
}

}  // namespace fq
