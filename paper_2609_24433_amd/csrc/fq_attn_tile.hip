// Attention for many query rows: a workgroup of four or eight waves holds 128 or 256 rows of one
// key head (32 a wave) and walks the keys in tiles of 64 that all its waves read from LDS.
//
// A tile costs a wave about as many cycles of the vector unit (exponentials, conversion of codes) as
// of the matrix unit, and a wave's vector instructions run while a matrix instruction of its own
// does.  So the loop is a pipeline over half tiles u of 32 keys, written as two chains of matrix
// instructions with a piece of vector work after each:
//   K Q^T of u + 1     with  the weights (exponentials) of u
//   V^T P^T of u       with  the last weights of u, the maxima of u + 1 and the staging of a tile's
//                            values (first half: of the next tile) or keys (second: the one after)
// Loads run a tile ahead of the staging.
//
// Measured, with the join: 4096 tokens over 8190 in the cache, causal, 32 query heads on 8 of 128: 400 to
// 434 us by the card, 1.0 PFLOP/s, 0.8 of what a plain product of 8192^3 reaches, the matrix units busy for
// 0.45 of the time under counters (on a card where it takes 422 us, 361 without loads and staging); 4 samples of 1031 queries over up to 4099 masked
// bf16 states, 16 heads on 8 of 128: 148 us, as long as its two long samples (4099 and 3514 states) take
// alone: their 144 workgroups run with the rest of the card idle.  Heads above 128 run one wave a SIMD: 4096
// causal tokens, 8 query heads on one of 256, 150 us, 0.46 PFLOP/s, and 816 tokens 30 us.
#include "fq_attn_device.hpp"
#include "fq_attn_launch.hpp"

namespace fq {
namespace {

constexpr int kTile = 64;

// LDS of a tile: keys [64][DP] bf16, the 16-byte pieces of a token's row swizzled; values
// transposed [DP][64 + 8] (cache) or [64][DP + 32] (states, read with the transposing read).  16
// lanes of a 16-byte access, and 32 of an 8-byte one, meet all 64 banks once.
template <bool CACHED, int DP>
struct Lds {
  static constexpr int kKeys = kTile * DP * 2;
  static constexpr int kVStride = CACHED ? 2 * kTile + 16 : 2 * DP + 64;  // bytes of a row
  static constexpr int kValues = (CACHED ? DP : kTile) * kVStride;
  static constexpr int kBytes = 2 * (kKeys + kValues) + (CACHED ? 0 : 4 * kTile * 4);
};
// 16 lanes read one piece of tokens 0-7 and 16-23 (or 8-15 and 24-31).
template <int DP>
__device__ __forceinline__ int swizzle(int token) {
  return DP == 64 ? ((token >> 1) & 3) | ((token >> 2) & 4) : (token & 7) | ((token >> 1) & 8);
}

template <bool CACHED, int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP < 256 ? 2 : 1) void attention_tile_kernel(AttnArgs a, Split sp, int row_tiles) {
  extern __shared__ __align__(16) uint8_t lds[];
  using L = Lds<CACHED, DP>;
  constexpr int kThreads = 64 * WAVES, kRows = 32 * WAVES;
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
  const int total = rows.n * G, r0 = tile_row * kRows;
  if (r0 >= total) return;

  // keys of the workgroup: its range, up to what its last row sees
  const int last_row = total - r0 > kRows ? r0 + kRows - 1 : total - 1;
  const int c0 = part * sp.chunk;
  int c1 = rows.end(last_row / G);
  if (c1 - c0 > sp.chunk) c1 = c0 + sp.chunk;
  if (c1 <= c0 && part > 0) return;  // no row of it has a partial result here
  const int tiles = c1 > c0 ? (c1 - c0 + kTile - 1) / kTile : 0;

  // this lane's row, as the column of both products
  const int b0 = r0 + wave * 32, row = b0 + col;
  const bool live = row < total;
  const int qi = live ? row / G : 0;
  const int hq = h * G + (live ? row - qi * G : 0);
  const int end = live ? rows.end(qi) : 0;
  const int least = b0 < total ? rows.end(b0 / G) : 0;  // that any row of the wave sees
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

  f32x16 o[DP / 32];
#pragma unroll
  for (int i = 0; i < DP / 32; ++i) o[i] = f32x16{};
  float m = -FLT_MAX, l[2] = {0.0f, 0.0f};  // l: of even and odd tokens
  const float c_all = a.scale * 1.4426950408889634f;

  // Loads of the tiles to come.  Every load is unconditional, at an address that is there (channels
  // from D on and tokens past the last one repeat others): what such places hold is finite or
  // replaced, meets zeros of q or weights of zero, or goes to channels nobody reads.
  struct Loaded {
    uint4 k[CACHED ? KU : VU], v[VU];
    float ks, vs;  // scales of 16-token group lane % 4
    uint32_t mask;
  };
  Loaded in, hold;  // in flight; of the tiles to stage
  const int last_key = rows.keys - 1;
  // A cache's tile is four 16-token groups, each in a page of its own perhaps: lane % 4 finds its
  // group's page, offset and scales, and a load takes its group's offset from that lane (the group
  // of a unit is the same for a whole wave, and so is the unit's place in it for all units).
  const int lp = CACHED ? 31 - __builtin_clz(a.c.P) : 0;
  const int32_t *pt = CACHED ? a.b.pt + s * a.b.width : nullptr;
  const int page_limit = CACHED ? (int)(a.c.pages - 1) : 0;
  const uint32_t head_bytes = CACHED ? a.c.P * D : 0, in_page = a.c.P - 1;
  const int8_t *kc = a.c.kc, *vc = a.c.vc;
  const uint32_t key_place = (tid / (DP / 16) % 16) * D + 16 * (16 * (tid % (DP / 16)) < D ? tid % (DP / 16) : 0);
  const uint32_t value_place = 16 * (tid % DP < D ? tid % DP : 0);
  int page_next = 0;                  // looked up a tile ahead
  int64_t at_k = 0, at_v = 0;         // byte offset of the group in the codes
  int64_t scale_k = 0, scale_v = 0;   // index of its scales
  auto look_up = [&](int t) {
    const int j = c0 + t * kTile + 16 * (lane & 3);
    page_next = pt[(j < last_key ? j : last_key) >> lp];
  };
  auto find = [&](int t) {
    const int page = page_next < 0 ? 0 : page_next > page_limit ? page_limit : page_next;
    scale_k = (int64_t)page * a.c.H + h;
    at_k = scale_k * head_bytes + (uint32_t)(((c0 + t * kTile + 16 * (lane & 3)) & in_page) * D);
  };
  auto group_at = [&](int64_t at, int g) {
    const uint32_t lo = __builtin_amdgcn_readlane((uint32_t)at, g), hi = __builtin_amdgcn_readlane((uint32_t)(at >> 32), g);
    return (int64_t)((uint64_t)hi << 32 | lo);
  };
  // States: a thread's places in a tile (bytes; the last tile's stop at the last state).
  const uint16_t *kp = a.k.p + s * a.k.bs + h * a.k.hs, *vp = a.v.p + s * a.v.bs + h * a.v.hs;
  uint32_t off_k[CACHED ? 1 : VU], off_v[CACHED ? 1 : VU];
  auto places = [&](int last, int64_t ts, uint32_t(&off)[CACHED ? 1 : VU]) {
    if constexpr (!CACHED)
#pragma unroll
      for (int i = 0; i < VU; ++i) {
        const int u = tid + i * kThreads, tk = u / (DP / 8), piece = 8 * (u % (DP / 8));
        off[i] = 2 * ((uint32_t)(tk < last ? tk : last) * (uint32_t)ts + (piece < D ? piece : 0));
      }
  };
  places(kTile - 1, a.k.ts, off_k);
  places(kTile - 1, a.v.ts, off_v);
  auto load_keys = [&](int t) {
    if constexpr (CACHED) {
      find(t);
#pragma unroll
      for (int i = 0; i < KU; ++i) {
        const int g = __builtin_amdgcn_readfirstlane((tid + i * kThreads) / DP);
        in.k[i] = *reinterpret_cast<const uint4 *>(kc + group_at(at_k, g) + key_place);
      }
      in.ks = a.c.ks[scale_k];
    } else {
      const int j0 = c0 + t * kTile, last = last_key - j0;
      if (last < kTile - 1) places(last < 0 ? 0 : last, a.k.ts, off_k);
      const char *base = reinterpret_cast<const char *>(kp + (int64_t)(last < 0 ? last_key : j0) * a.k.ts);
#pragma unroll
      for (int i = 0; i < VU; ++i) in.k[i] = *reinterpret_cast<const uint4 *>(base + off_k[i]);
    }
  };
  auto load_values = [&](int t) {
    if constexpr (CACHED) {
#pragma unroll
      for (int i = 0; i < VU; ++i) {
        const int g = __builtin_amdgcn_readfirstlane((tid + i * kThreads) / DP);
        in.v[i] = *reinterpret_cast<const uint4 *>(vc + group_at(at_v, g) + value_place);
      }
      in.vs = a.c.vs[scale_v];
    } else {
      const int j0 = c0 + t * kTile, last = last_key - j0;
      if (last < kTile - 1) places(last < 0 ? 0 : last, a.v.ts, off_v);
      const char *base = reinterpret_cast<const char *>(vp + (int64_t)(last < 0 ? last_key : j0) * a.v.ts);
#pragma unroll
      for (int i = 0; i < VU; ++i) in.v[i] = *reinterpret_cast<const uint4 *>(base + off_v[i]);
    }
  };
  // One place of a tile a lane: whether its state is seen.
  auto load_mask = [&](int t) {
    if constexpr (!CACHED) {
      const int j = c0 + t * kTile + lane;
      in.mask = j <= last_key;
      if (a.mask) in.mask &= a.mask[s * a.mask_stride + (j <= last_key ? j : last_key)] != 0;
    }
  };
  // Tile t's loads: its values, and the keys and the mask of the tile after it.
  auto load = [&](int t) {
    load_values(t);
    load_keys(t + 1);
    load_mask(t + 1);
    at_v = at_k;
    scale_v = scale_k;
    if constexpr (CACHED) look_up(t + 2);
  };

  uint8_t *const keys_at = lds, *const values_at = lds + 2 * L::kKeys;
  // Staging in pieces, 8 channels (tokens) of a unit each: the held keys go to buffer kb, the values
  // to buffer vb.
  constexpr int kKeyPieces = CACHED ? 2 * KU : VU, kValuePieces = CACHED ? 2 * VU : VU;
  using KeyPieces = std::integral_constant<int, kKeyPieces>;
  using ValuePieces = std::integral_constant<int, kValuePieces>;
  auto stage_key = [&](uint8_t *to, int n) {
    if constexpr (CACHED) {
      const int i = n / 2, e = n % 2;
      const int u = tid + i * kThreads, tk = u / (DP / 16), piece = 2 * (u % (DP / 16)) + e;
      *reinterpret_cast<uint4 *>(to + tk * DP * 2 + ((piece ^ swizzle<DP>(tk)) * 16)) =
          e == 0 ? codes8_to_bf16(hold.k[i].x, hold.k[i].y) : codes8_to_bf16(hold.k[i].z, hold.k[i].w);
    } else {
      const int u = tid + n * kThreads, tk = u / (DP / 8), piece = u % (DP / 8);
      *reinterpret_cast<uint4 *>(to + tk * DP * 2 + ((piece ^ swizzle<DP>(tk)) * 16)) = hold.k[n];
    }
  };
  auto stage_value = [&](uint8_t *to, int n) {
    if constexpr (CACHED) {
      const int j = n / 2, e = n % 2;
      const int u = tid + j * kThreads, d = u % DP, g = u / DP;
      *reinterpret_cast<uint4 *>(to + d * L::kVStride + g * 32 + 16 * e) =
          e == 0 ? codes8_to_bf16(hold.v[j].x, hold.v[j].y) : codes8_to_bf16(hold.v[j].z, hold.v[j].w);
    } else {
      const int u = tid + n * kThreads, tk = u / (DP / 8), piece = u % (DP / 8);
      *reinterpret_cast<uint4 *>(to + tk * L::kVStride + piece * 16) = hold.v[n];
    }
  };
  // Unseen states: zeros for their keys and values (they may hold anything), zeros for channels from
  // D on, and minus infinity where a tile's scores start from (one of four buffers).
  float *const bias = reinterpret_cast<float *>(lds + 2 * (L::kKeys + L::kValues));
  auto clear_rows = [&](uint4(&x)[VU], uint64_t seen) {
    if (!CACHED && (D < DP || seen != ~0ull))
#pragma unroll
      for (int i = 0; i < VU; ++i) {
        const int u = tid + i * kThreads, tk = u / (DP / 8), piece = 8 * (u % (DP / 8));
        if (piece >= D || !(seen >> tk & 1)) x[i] = make_uint4(0, 0, 0, 0);
      }
  };
  auto write_bias = [&](int t) {
    if (!CACHED && wave == 0) bias[(t & 3) * kTile + lane] = hold.mask ? 0.0f : -INFINITY;
  };

  // S^T: row i = 8 x + 4 y + z of a 32-token block is token 16 y + 4 x + z
  const int token = 16 * ((col >> 2) & 1) + 4 * (col >> 3) + (col & 3), sw = swizzle<DP>(token);
  constexpr int STEPS = DP / 16;  // operands of a half tile, of either product
  constexpr int AHEAD = 3;        // operands read ahead of the instructions that use them
  // Keys' operand n of half b: channels 16 n ..; values' operand n: channels 32 (n % (DP/32)) .., step
  // n / (DP/32) of 16 tokens, where a lane's are 32 b + 16 half + 8 step ..
  auto key_operand = [&](const uint8_t *kb, int b, int n) {
    return *reinterpret_cast<const uint4 *>(kb + (32 * b + token) * DP * 2 + (((2 * n + half) ^ sw) * 16));
  };
  auto value_operand = [&](const uint8_t *vb, int b, int n) {
    const int i = n % (DP / 32), x = n / (DP / 32);
    if constexpr (CACHED) {
      return *reinterpret_cast<const uint4 *>(vb + (32 * i + col) * L::kVStride + (32 * b + 16 * half + 8 * x) * 2);
    } else {
      const int piece = lane % 16;
      const uint8_t *at = vb + (32 * b + 16 * half + 8 * x + piece / 4) * L::kVStride +
                          (32 * i + 16 * ((lane >> 4) & 1) + 4 * (piece % 4)) * 2;
      const uint2 v0 = lds_read_transposed(at), v1 = lds_read_transposed(at + 4 * L::kVStride);
      return make_uint4(v0.x, v0.y, v1.x, v1.y);
    }
  };
  // STEPS operands and products, with `work` (step) behind each matrix instruction; the reads run on into the operands of the next chain.  The walls hold the order:
  // left alone the compiler reads all operands at once, for which there are no registers, or gathers
  // the vector work behind the products.
  uint4 ring[AHEAD + 1];
  static_assert(STEPS % (AHEAD + 1) == 0, "a chain leaves the ring where the next one starts");
  auto prime = [&](auto operand) {
#pragma unroll
    for (int n = 0; n < AHEAD; ++n) ring[n] = operand(n);
  };
  auto chain = [&](auto operand, auto next_operand, auto product, auto work) {
    sched_wall();
    auto step = [&](auto at) {
      constexpr int n = decltype(at)::value;
      ring[(n + AHEAD) % (AHEAD + 1)] = n + AHEAD < STEPS ? operand(n + AHEAD) : next_operand(n + AHEAD - STEPS);
      product(n, __builtin_bit_cast(bf16x8, ring[n % (AHEAD + 1)]));
      work(at);
      sched_wall();
    };
    static_for<STEPS>(step);
  };
  // f(i) for the part of `count` pieces, spread over instructions [from, until) of a chain, that
  // belongs to instruction `at`
  auto share = [](auto at, int from, int until, int count, auto f) {
    const int n = decltype(at)::value, N = until - from;
    if (n < from || n >= until) return;
#pragma unroll
    for (int i = (n - from) * count / N; i < (n - from + 1) * count / N; ++i) f(i);
  };

  // Scores of a half tile: a lane has 16 tokens of one 16-token group, with one scale c.  States'
  // scores start from their bias.  Where a cache's tokens lie beyond the row's end they become
  // -infinity, with the scale applied here, so that a scale that is 0 or NaN reaches only what is
  // seen; a NaN scale of the values goes by the scores.
  struct Scores {
    f32x16 st;
    float c, v, top;
  };
  auto begin = [&](Scores &z, int t, int b, float ks, float vs) {
    if constexpr (CACHED) {
      z.st = f32x16{};
    } else {
      const float4 *p = reinterpret_cast<const float4 *>(bias + (t & 3) * kTile + 32 * b + 16 * half);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float4 f = p[e];
        z.st[4 * e] = f.x, z.st[4 * e + 1] = f.y, z.st[4 * e + 2] = f.z, z.st[4 * e + 3] = f.w;
      }
    }
    z.c = CACHED ? c_all * ks : c_all;
    z.v = CACHED ? vs : 1.0f;
  };
  auto hide_unseen = [&](Scores &z, int t, int b) {
    const int j0 = c0 + t * kTile + 32 * b;
    if (CACHED && j0 + 32 > least) {
      const int left = end - (j0 + 16 * half);
      const uint32_t on = left >= 16 ? 0xFFFFu : left <= 0 ? 0u : (1u << left) - 1;
      const float bad = z.v - z.v;
#pragma unroll
      for (int e = 0; e < 16; ++e) z.st[e] = (on >> e & 1) ? __builtin_fmaf(z.st[e], z.c, bad) : -INFINITY;
      z.c = 1.0f;
      z.v = bad == 0.0f ? z.v : 1.0f;
    }
  };
  // maximum of a lane's scores, two at a time: piece n of 8
  auto two_maxima = [&](Scores &z, int n) {
    const float t0 = maxf(z.st[2 * n], z.st[2 * n + 1]);
    z.top = n == 0 ? t0 : maxf(z.top, t0);
    asm volatile("" : "+v"(z.top));
  };
  // The running maximum moves only where it has to: a weight up to 2^8 is as exact as one up to 1.
  auto follow_maximum = [&](const Scores &z) {
    const float top = z.top * z.c;
    if (__any(top > m + 8.0f)) {
      const float to = maxf(m, across32(maxf(top, -FLT_MAX), maxf)), shrink = exp2_fast(m - to);
      m = to;
      l[0] *= shrink;
      l[1] *= shrink;
#pragma unroll
      for (int i = 0; i < DP / 32; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] *= shrink;
    }
  };
  uint4 w[2];  // weights in the operand order of the second product
  // Two scores to weights: piece n of 8 + 1.  The exponentials of a piece come with the sums and
  // conversions of the one before, whose results they would otherwise wait for.
  float e0 = 0.0f, e1 = 0.0f;
  auto two_weights = [&](const Scores &z, int n) {
    const float p0 = e0, p1 = e1;
    if (n < 8) {
      e0 = exp2_fast(__builtin_fmaf(z.st[2 * n], z.c, -m));
      e1 = exp2_fast(__builtin_fmaf(z.st[2 * n + 1], z.c, -m));
    }
    if (n > 0) {
      const int y = n - 1;
      // Weights enter the product as bf16, with the scale of the values in them: 9 bits of each, as the
      // result will have.  What the rounding drops would take a second product, and matrix instructions
      // bound the kernel.
      uint32_t u;
      if constexpr (CACHED) {
        l[0] += p0;
        l[1] += p1;
        u = pack_bf16(p0 * z.v, p1 * z.v);
      } else {  // the sum of the weights as they are used
        u = pack_bf16(p0, p1);
        l[n % 2] = add_pair(u, l[n % 2]);
      }
      asm volatile("" : "+v"(u), "+v"(l[0]), "+v"(l[1]));  // here, not where the weights are used
      uint4 &to = w[y / 4];
      (y % 4 == 0 ? to.x : y % 4 == 1 ? to.y : y % 4 == 2 ? to.z : to.w) = u;
    }
    asm volatile("" : "+v"(e0), "+v"(e1));
  };
  auto output_product = [&](int n, bf16x8 u) {
    const int i = n % (DP / 32);
    o[i] = mfma32(u, __builtin_bit_cast(bf16x8, w[n / (DP / 32)]), o[i]);
  };
  constexpr int kWeights = 9, kMaxima = 8;
  // weights left for the first half of the second chain, whose products need only the first half
  constexpr int kLate = kWeights * 5 / 16;

  // Weights and outputs of a half tile (b of values vb), scores of the next (b_next of tile t_next:
  // keys kb; after it, operands from `following`), with `pieces` of staging in the second chain.
  auto half_tile = [&](Scores &now, Scores &next, const uint8_t *vb, int b, const uint8_t *kb, int t_next, int b_next,
                       auto following, auto pieces, auto stage) {
    auto values = [&](int n) { return value_operand(vb, b, n); };
    chain([&](int n) { return key_operand(kb, b_next, n); }, values,
          [&](int n, bf16x8 k) { next.st = mfma32(k, q[n], next.st); },
          [&](auto at) { share(at, 0, STEPS, kWeights - kLate, [&](int n) { two_weights(now, n); }); });
    hide_unseen(next, t_next, b_next);
    chain(values, following, output_product, [&](auto at) {
      share(at, 0, STEPS / 2, kLate, [&](int n) { two_weights(now, kWeights - kLate + n); });
      share(at, STEPS / 8, STEPS, kMaxima, [&](int n) { two_maxima(next, n); });
      share(at, STEPS / 2, STEPS, decltype(pieces)::value, stage);
    });
    follow_maximum(next);
  };

  // scale of a lane's half of the tokens of half tile b, from the lanes that hold the groups' scales
  auto scale_of = [&](float v, int b) {
    const float x0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 2 * b));
    const float x1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), 2 * b + 1));
    return half ? x1 : x0;
  };
  Scores sa, sb;
  float ks0 = 0.0f, ks1 = 0.0f, vs0 = 0.0f, vs1 = 0.0f;  // scales of this tile's groups and the next's
  auto bits_of = [&](uint32_t mask) { return CACHED ? ~0ull : __ballot(mask != 0); };
  uint64_t bits = ~0ull;  // seen places of the tile after this one
  uint64_t seen = 0;      // of all tiles
  if (tiles > 0) {
    // keys 0 and 1 and values 0 into LDS, values 1 and keys 2 under way
    if constexpr (CACHED) look_up(0);
    load_keys(0);
    load_mask(0);
    at_v = at_k;
    scale_v = scale_k;
    if constexpr (CACHED) look_up(1);
#pragma unroll
    for (int i = 0; i < (CACHED ? KU : VU); ++i) hold.k[i] = in.k[i];
    hold.mask = in.mask;
    ks0 = in.ks;
    load(0);
    const uint64_t bits0 = bits_of(hold.mask);
    write_bias(0);
    if constexpr (!CACHED) clear_rows(hold.k, bits0);
#pragma unroll
    for (int n = 0; n < kKeyPieces; ++n) stage_key(keys_at, n);
    hold = in;
    bits = bits_of(hold.mask);
    seen = bits0 | bits;
    ks1 = in.ks;
    vs0 = in.vs;
    load(1);
    write_bias(1);
    if constexpr (!CACHED) {
      clear_rows(hold.k, bits);
      clear_rows(hold.v, bits0);
    }
#pragma unroll
    for (int n = 0; n < kKeyPieces; ++n) stage_key(keys_at + L::kKeys, n);
#pragma unroll
    for (int n = 0; n < kValuePieces; ++n) stage_value(values_at, n);
    __syncthreads();
    begin(sa, 0, 0, scale_of(ks0, 0), scale_of(vs0, 0));
    auto first = [&](int n) { return key_operand(keys_at, 0, n); };
    prime(first);
    chain(first, [&](int n) { return key_operand(keys_at, 1, n); },
          [&](int n, bf16x8 k) { sa.st = mfma32(k, q[n], sa.st); }, [](auto) {});
    hide_unseen(sa, 0, 0);
#pragma unroll
    for (int n = 0; n < kMaxima; ++n) two_maxima(sa, n);
    follow_maximum(sa);
  }
  // Tile t, with its buffers known to the compiler.
  auto tile = [&](int t, auto parity) {
    constexpr int even = decltype(parity)::value;
    // values t and keys t + 1 are in LDS (behind the barrier), values t + 1 and keys t + 2 under way
    const uint8_t *vb = values_at + even * L::kValues;
    uint8_t *k0 = keys_at + even * L::kKeys, *k1 = keys_at + (1 - even) * L::kKeys;
    __syncthreads();
    begin(sb, t, 1, scale_of(ks0, 1), scale_of(vs0, 1));
    hold = in;
    load(t + 2);
    write_bias(t + 2);
    if constexpr (!CACHED) {
      clear_rows(hold.v, bits);
      bits = bits_of(hold.mask);
      seen |= bits;
      clear_rows(hold.k, bits);
    }
    half_tile(sa, sb, vb, 0, k0, t, 1, [&](int n) { return key_operand(k1, 0, n); }, ValuePieces{},
              [&](int n) { stage_value(values_at + (1 - even) * L::kValues, n); });
    vs1 = hold.vs;
    __syncthreads();
    begin(sa, t + 1, 0, scale_of(ks1, 0), scale_of(vs1, 0));
    half_tile(sb, sa, vb, 1, k1, t + 1, 0, [&](int n) { return key_operand(k1, 1, n); }, KeyPieces{},
              [&](int n) { stage_key(k0, n); });
    ks0 = ks1, vs0 = vs1, ks1 = hold.ks;
  };
  for (int t = 0; t < tiles; t += 2) {
    tile(t, std::integral_constant<int, 0>{});
    if (t + 1 == tiles) break;
    tile(t + 1, std::integral_constant<int, 1>{});
  }
  // Where nothing is seen the results are zeros, also for a query that is not finite, whose products with the
  // zeros of unseen places are not.  (`seen` has tiles behind this part's too: where those hold the only seen
  // places, another part has them and such a query's row is NaN as it should be.)
  if (!CACHED && seen == 0) {
    l[0] = l[1] = 0.0f;
#pragma unroll
    for (int i = 0; i < DP / 32; ++i) o[i] = f32x16{};
  }
  const float sum = across32(l[0] + l[1], [](float y, float z) { return y + z; });
  if (!live) return;
  // a lane holds channels 32 i + 8 y + 4 half + z of its row
  if (sp.splits > 1) {
    const int64_t at = (((int64_t)part * a.seqs + s) * a.Hk + h) * (a.max_new * G) + row;
    if (half == 0) sp.ml[at] = make_float2(m, sum);
#pragma unroll
    for (int i = 0; i < DP / 32; ++i)
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int d = 32 * i + 8 * y + 4 * half;
        if (d < D)
          *reinterpret_cast<float4 *>(sp.o + at * D + d) = make_float4(o[i][4 * y], o[i][4 * y + 1], o[i][4 * y + 2], o[i][4 * y + 3]);
      }
    return;
  }
  const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
  uint16_t *out = a.out + ((rows.q0 + qi) * a.Hq + hq) * D;
#pragma unroll
  for (int i = 0; i < DP / 32; ++i)
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const int d = 32 * i + 8 * y + 4 * half;
      if (d < D)
        *reinterpret_cast<uint2 *>(out + d) = make_uint2(pack_bf16(o[i][4 * y] * inv, o[i][4 * y + 1] * inv),
                                                        pack_bf16(o[i][4 * y + 2] * inv, o[i][4 * y + 3] * inv));
    }
}

template <bool CACHED, int DP, int WAVES>
hipError_t launch(const AttnArgs &a, const Split &sp, hipStream_t s) {
  static std::atomic<uint64_t> raised{0};
  const size_t lds = Lds<CACHED, DP>::kBytes;
  hipError_t e = allow_dynamic_lds(attention_tile_kernel<CACHED, DP, WAVES>, lds, raised);
  if (e != hipSuccess) return e;
  const int rows = 32 * WAVES;
  const int64_t row_tiles = (a.max_new * (a.Hq / a.Hk) + rows - 1) / rows;
  attention_tile_kernel<CACHED, DP, WAVES>
      <<<dim3((unsigned)(a.Hk * row_tiles * sp.splits), (unsigned)a.seqs), 64 * WAVES, lds, s>>>(a, sp, (int)row_tiles);
  return hipGetLastError();
}

template <bool CACHED>
hipError_t launch_size(const AttnArgs &a, const Split &sp, int rows, hipStream_t s) {
  if (a.D <= 64) return launch<CACHED, 64, 4>(a, sp, s);
  if (a.D <= 128) return rows > 128 ? launch<CACHED, 128, 8>(a, sp, s) : launch<CACHED, 128, 4>(a, sp, s);
  return launch<CACHED, 256, 4>(a, sp, s);
}

}  // namespace

hipError_t launch_attention_tile(bool cached, const AttnArgs &a, const Split &sp, int rows, hipStream_t s) {
  return cached ? launch_size<true>(a, sp, rows, s) : launch_size<false>(a, sp, rows, s);
}

}  // namespace fq
