// Norms of queries and keys per head, the position rotation, and appends to the 8-bit cache.
//
// A head of D values is held by D/16 lanes of a group of L (the next power of two), 16 values a
// lane: the two 8-value chunks that the rotation pairs, dims [8m, 8m + 8) and the same R/2
// further on (halves), or 16 adjacent dims (adjacent pairs, and dims the rotation leaves alone).
// So a rotation never crosses lanes, and the only exchange is the norm's sum.  Norm and rotation are
// fp32 from the bf16 input to the one rounding at the end.
//
// All are bound by memory where they are long and by launches and the latency of dependent loads
// where they are short.  Measured: norm and rotation of 16385 tokens, 40 heads of 128: 74 to 79 us by the
// card (71 in a kernel trace), 4.3 to 4.6 TB/s; of 50 tokens, 9 heads of 256: 4.1 us.  Append of a prompt of 16383
// tokens, 32 query and 8 key heads of 128: 95 us, 4.3 TB/s; of one token to each of 32 sequences: 6.5 us where no
// page's scale grows, 8.4 where every page's does, most of it a page's chain of waits (lengths, table entry,
// scale, codes).  Read of the last page of each of 32 sequences: 8 us; of 16383 tokens, 8 heads of 128: 23 us, 4.3
// TB/s.
#include <cfloat>

#include "fq_attn.hpp"
#include "fq_device.hpp"

namespace fq {
namespace {

constexpr int kThreads = 256;

// Where a lane's 16 values of a head lie, and its part of the rotation.
struct Place {
  int a, b;  // first dims of its two chunks
  bool in, rot;
};
__device__ __forceinline__ Place place_of(int m, int D, int rot, int interleaved) {
  Place p;
  p.in = m < D / 16;
  p.rot = m < rot / 16;
  const bool halves = p.rot && !interleaved;
  p.a = halves ? 8 * m : 16 * m;
  p.b = halves ? 8 * m + rot / 2 : 16 * m + 8;
  return p;
}

__device__ __forceinline__ void unpack8(const uint4 &u, float *v) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = bf16_lo(w[i]);
    v[2 * i + 1] = bf16_hi(w[i]);
  }
}
__device__ __forceinline__ uint4 pack8(const float *v) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = f32_to_bf16(v[2 * i]) | (f32_to_bf16(v[2 * i + 1]) << 16);
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct Raw {
  uint4 a, b;
};
__device__ __forceinline__ Raw load_raw(const uint16_t *x, const Place &p, bool on) {
  Raw r{make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
  if (on && p.in) {
    r.a = *reinterpret_cast<const uint4 *>(x + p.a);
    r.b = *reinterpret_cast<const uint4 *>(x + p.b);
  }
  return r;
}
__device__ __forceinline__ void unpack(const Raw &r, float (&v)[16]) {
  unpack8(r.a, v);
  unpack8(r.b, v + 8);
}

__device__ __forceinline__ void load_weight(const float *w, const Place &p, float (&g)[16]) {
#pragma unroll
  for (int i = 0; i < 16; ++i) g[i] = 1.0f;
  if (w && p.in)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      g[i] = w[p.a + i];
      g[8 + i] = w[p.b + i];
    }
}

__device__ __forceinline__ void load_angles(const Rope &r, const Place &p, int m, int64_t position, float2 (&cs)[8]) {
  if (!p.rot) return;
  const int64_t at = position < 0 ? 0 : position >= r.length ? r.length - 1 : position;
  const float4 *t = reinterpret_cast<const float4 *>(r.table + at * (r.rot / 2) + 8 * m);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float4 f = t[i];
    cs[2 * i] = make_float2(f.x, f.y);
    cs[2 * i + 1] = make_float2(f.z, f.w);
  }
}

// Norm (w given) and rotation of one head.  The sum of squares is fp32: 16 values a lane in
// order, then a tree over the group's lanes.
template <int L>
__device__ __forceinline__ void norm_rotate(float (&v)[16], bool norm, const float (&g)[16], const float2 (&cs)[8],
                                            const Place &p, int interleaved, float eps, int D) {
  if (norm) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s = __builtin_fmaf(v[i], v[i], s);
#pragma unroll
    for (int d = 1; d < L; d *= 2) s += __shfl_xor(s, d);
    const float r = 1.0f / sqrtf(s / (float)D + eps);
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = v[i] * r * g[i];
  }
  if (!p.rot) return;
  auto turn = [&](float &a, float &b, float2 t) {
    const float x = a, y = b;
    a = __builtin_fmaf(x, t.x, -(y * t.y));
    b = __builtin_fmaf(y, t.x, x * t.y);
  };
  if (interleaved)
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(v[2 * i], v[2 * i + 1], cs[i]);
  else
#pragma unroll
    for (int i = 0; i < 8; ++i) turn(v[i], v[8 + i], cs[i]);
}

__device__ __forceinline__ void store_head(uint16_t *y, const Place &p, const float (&v)[16]) {
  if (!p.in) return;
  *reinterpret_cast<uint4 *>(y + p.a) = pack8(v);
  *reinterpret_cast<uint4 *>(y + p.b) = pack8(v + 8);
}

__global__ void rope_table_kernel(const double *__restrict__ f, double magnitude, int64_t length, int64_t pairs,
                                  float2 *__restrict__ table) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= length * pairs) return;
  double s, c;
  sincos((double)(i / pairs) * f[i % pairs], &s, &c);
  table[i] = make_float2((float)(magnitude * c), (float)(magnitude * s));
}

// One token's heads slice, slice + S, ... of H (S = H: one): its angles and weights stay in registers.
template <int L>
__device__ __forceinline__ void rope_heads(const uint16_t *x, int64_t hs, uint16_t *y, int H, int slice, int S,
                                           const Rope &r, const float *w, const Place &p, const float2 (&cs)[8], int D) {
  float g[16];
  load_weight(w, p, g);
  for (int h = slice; h < H; h += S) {
    float v[16];
    unpack(load_raw(x + h * hs, p, true), v);
    norm_rotate<L>(v, w != nullptr, g, cs, p, r.interleaved, r.eps, D);
    store_head(y + (int64_t)h * D, p, v);
  }
}

// Grid: units of (token, head), query heads before key heads.
template <int L>
__global__ __launch_bounds__(kThreads) void qk_rope_kernel(Heads q, int Hq, Heads k, int Hk, Rope r, int64_t T, int D,
                                                           uint16_t *__restrict__ q_out, uint16_t *__restrict__ k_out) {
  const int64_t u = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const int H = Hq + Hk, m = threadIdx.x % L;
  const int64_t t = u / H;
  if (t >= T) return;
  const int h = (int)(u - t * H);
  const Place p = place_of(m, D, r.rot, r.interleaved);
  float2 cs[8];
  load_angles(r, p, m, r.positions ? r.positions[t] : t, cs);
  if (h < Hq)
    rope_heads<L>(q.p + t * q.ts, q.hs, q_out + t * Hq * D, Hq, h, Hq, r, r.qw, p, cs, D);
  else
    rope_heads<L>(k.p + t * k.ts, k.hs, k_out + t * Hk * D, Hk, h - Hq, Hk, r, r.kw, p, cs, D);
}

// ---------------------------------------------------------------- appends

// The rows of sequence s that this call computes: [row, row + n), and their slots [begin, end).  All the
// sequence's rows count for the slot of the first one, those past max_new too: row i goes to slot kv_len - rows + i
// (which is negative where kv_len is short: such rows are dropped).
struct Span1 {
  int64_t row;
  int n;
  int64_t begin, end;
};
__device__ __forceinline__ Span1 sequence_rows(const Batch &b, int64_t s, int64_t T) {
  Span1 r;
  int64_t q0 = b.q_start[s], q1 = b.q_start[s + 1];
  q0 = q0 < 0 ? 0 : q0 > T ? T : q0;
  q1 = q1 < q0 ? q0 : q1 > T ? T : q1;
  const int64_t n = q1 - q0 < b.max_new ? q1 - q0 : b.max_new;
  const int64_t m = b.kv_len[s];
  r.row = q0;
  r.n = (int)n;
  r.begin = m - (q1 - q0);
  r.end = r.begin + n < b.max_kv ? r.begin + n : b.max_kv;
  return r;
}

__device__ __forceinline__ int64_t page_of(const Batch &b, int64_t pages, int64_t s, int64_t w) {
  const int64_t p = b.pt[s * b.width + w];
  return p < 0 ? 0 : p >= pages ? pages - 1 : p;
}

// |x| as an integer: orders like |x|, with infinity and NaN above every finite value.
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7FFFFFFFu; }

__device__ __forceinline__ int code_of(float x, float inv) {
  return (int)__builtin_rintf(__builtin_amdgcn_fmed3f(x * inv, -127.0f, 127.0f));
}

// Four earlier codes at the grown scale.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float ratio) {
  uint32_t r = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float c = (float)(int8_t)(w >> (8 * i));
    r |= ((uint32_t)(int)__builtin_rintf(c * ratio) & 0xFFu) << (8 * i);
  }
  return r;
}

__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t *lds) {
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const uint32_t o = (uint32_t)__shfl_xor((int)v, d);
    v = o > v ? o : v;
  }
  if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int i = 1; i < kThreads / 64; ++i) v = lds[i] > v ? lds[i] : v;
  return v;
}

// Workgroups [0, kv_items): one page of one sequence and head, keys or values.  The page's new tokens
// are read once, NP a lane group, and stay in registers as they came: their largest value gives the
// scale, then they become codes.  A scale that has to grow grows by c.growth at least: each growth rounds the
// earlier codes once more, and codes that a ratio near 1 leaves as they are drift with the scale.  The other
// workgroups: the query heads of the new tokens.
template <int L, int NP>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(Cache c, Batch b, Heads k, Heads v, Heads q, int Hq,
                                                                int Sq, int64_t kv_items, int pages_per_seq,
                                                                int64_t q_blocks, Rope r, int64_t T,
                                                                uint16_t *__restrict__ q_out) {
  // values: the page's new codes [P/16][D][16], 16 bytes more every 16 channels (a token's channels
  // are written 16 apart by the lanes: the gap moves them to banks of their own)
  extern __shared__ __align__(16) uint8_t tile[];
  __shared__ uint32_t red[kThreads / 64];
  constexpr int NG = kThreads / L;
  const int D = c.D, P = c.P, m = threadIdx.x % L, grp = threadIdx.x / L;
  const Place p = place_of(m, D, r.rot, r.interleaved);
  if ((int64_t)blockIdx.x >= kv_items) {
    const int64_t x = (int64_t)blockIdx.x - kv_items, s = x / q_blocks;
    const Span1 sp = sequence_rows(b, s, T);
    const int64_t u = (x - s * q_blocks) * NG + grp;
    const int64_t i = u / Sq;
    if (i >= sp.n) return;
    const int64_t t = sp.row + i;
    float2 cs[8];
    load_angles(r, p, m, r.positions ? r.positions[t] : sp.begin + i, cs);
    rope_heads<L>(q.p + t * q.ts, q.hs, q_out + t * Hq * D, Hq, (int)(u - i * Sq), Sq, r, r.qw, p, cs, D);
    return;
  }
  const bool keys = (blockIdx.x & 1) == 0;
  const int64_t item = blockIdx.x >> 1;
  const int h = (int)(item % c.H);
  const int64_t s = item / c.H / pages_per_seq;
  const Span1 sp = sequence_rows(b, s, T);
  const int64_t first = sp.begin > 0 ? sp.begin : 0;
  const int64_t pw = first / P + item / c.H % pages_per_seq, lo = pw * P;
  const int64_t s0 = lo > first ? lo : first, s1 = lo + P < sp.end ? lo + P : sp.end;
  if (sp.n <= 0 || s1 <= s0) return;
  const int held = (int)(first > lo ? first - lo : 0), from = (int)(s0 - lo), to = (int)(s1 - lo);
  const int64_t page = page_of(b, c.pages, s, pw) * c.H + h;
  const Place pl = keys ? p : place_of(m, D, 0, 0);
  float *scale_at = (keys ? c.ks : c.vs) + page;
  const float old = held ? *scale_at : 0.0f;
  const int64_t t0 = sp.row + (s0 - sp.begin);  // token of slot s0
  const Heads &in = keys ? k : v;
  Raw raw[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int o = grp + i * NG;
    raw[i] = load_raw(in.p + (t0 + o) * in.ts + h * in.hs, pl, from + o < to);
  }
  float g[16];
  load_weight(keys ? r.kw : nullptr, pl, g);
  auto value = [&](int i, float(&x)[16]) {
    unpack(raw[i], x);
    const int o = grp + i * NG;
    if (keys && from + o < to) {
      float2 cs[8];
      load_angles(r, pl, m, r.positions ? r.positions[t0 + o] : s0 + o, cs);
      norm_rotate<L>(x, r.kw != nullptr, g, cs, pl, r.interleaved, r.eps, D);
    }
  };

  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    float x[16];
    value(i, x);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const uint32_t a = abs_bits(x[e]);
      top = a > top ? a : top;
    }
  }
  top = block_max(top, red);  // every thread has read the old scale
  float scale = __uint_as_float(top) / 127.0f;
  bool bad = top >= 0x7F800000u;
  if (held) {
    bad = bad || old != old;
    scale = old >= scale ? old : __builtin_fmaxf(scale, old * c.growth);
  }
  if (!(scale >= FLT_MIN)) scale = 0.0f;
  const bool grew = held && !bad && scale != old;
  const float inv = scale > 0.0f && !bad ? 1.0f / scale : 0.0f;
  const float ratio = scale > 0.0f ? old / scale : 0.0f;
  if (threadIdx.x == 0) *scale_at = bad ? __uint_as_float(0x7FC00000u) : scale;

  if (keys) {
    int8_t *base = c.kc + page * P * D;
    if (grew)
      for (int i = threadIdx.x; i < held * D / 16; i += kThreads) {
        uint4 *w = reinterpret_cast<uint4 *>(base) + i;
        const uint4 o = *w;
        *w = make_uint4(rescale4(o.x, ratio), rescale4(o.y, ratio), rescale4(o.z, ratio), rescale4(o.w, ratio));
      }
#pragma unroll
    for (int i = 0; i < NP; ++i) {
      const int o = from + grp + i * NG;
      if (o >= to) continue;
      float x[16];
      value(i, x);
      if (!pl.in) continue;  // (after the norm's exchange)
      uint32_t w[4] = {0, 0, 0, 0};
      if (!bad)
#pragma unroll
        for (int e = 0; e < 16; ++e) w[e / 4] |= ((uint32_t)code_of(x[e], inv) & 0xFFu) << (8 * (e % 4));
      int8_t *row = base + o * D;
      *reinterpret_cast<uint2 *>(row + pl.a) = make_uint2(w[0], w[1]);
      *reinterpret_cast<uint2 *>(row + pl.b) = make_uint2(w[2], w[3]);
    }
    return;
  }
  const int group_bytes = 17 * D;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int o = from + grp + i * NG;
    if (o >= to || !pl.in) continue;
    float x[16];
    value(i, x);
    uint8_t *at = tile + (o / 16) * group_bytes + m * 272 + o % 16;
#pragma unroll
    for (int e = 0; e < 16; ++e) at[16 * e] = bad ? 0 : (uint8_t)code_of(x[e], inv);
  }
  __syncthreads();
  // 16 tokens of one channel an item: earlier codes, then the new ones, then zeros
  const int g0 = grew ? 0 : from / 16, g1 = (to + 15) / 16;
  uint4 *base = reinterpret_cast<uint4 *>(c.vc + page * P * D);
  for (int i = g0 * D + threadIdx.x; i < g1 * D; i += kThreads) {
    const int group = i / D, d = i - group * D, t = group * 16;
    uint32_t w[4] = {0, 0, 0, 0};
    if (t < held) {
      const uint4 o = base[i];
      w[0] = o.x, w[1] = o.y, w[2] = o.z, w[3] = o.w;
      if (grew)
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = rescale4(w[j], ratio);
    }
    const uint4 n = *reinterpret_cast<const uint4 *>(tile + group * group_bytes + d * 16 + d / 16 * 16);
    const uint32_t nw[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int o = t + 4 * j + e;
        const uint32_t mask = 0xFFu << (8 * e);
        if (o >= from) w[j] = (w[j] & ~mask) | (o < to ? nw[j] & mask : 0u);
      }
    base[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// 64 tokens of one head: codes times scales, the rows of [first, last), zeros beyond.  All of a
// thread's loads (NJ pieces of 8 channels, NJ / 2 of 16 tokens) are in flight together: the kernel
// waits three times on memory, for the bounds, the pages and the codes, whatever it moves.
constexpr int kReadTokens = 64;
template <int NJ>
__global__ __launch_bounds__(kThreads) void cache_read_kernel(Cache c, const int32_t *__restrict__ pt, int64_t width,
                                                              const int32_t *__restrict__ first,
                                                              const int32_t *__restrict__ last, int windows,
                                                              int64_t max_tokens, uint16_t *__restrict__ k_out,
                                                              uint16_t *__restrict__ v_out) {
  // values [4][D][16], 16 bytes more every 8 channels: lanes that read a token's channels, 8 apart,
  // meet banks of their own
  __shared__ __align__(16) uint8_t vt[kReadTokens / 16 * 18 * 32 * NJ];
  __shared__ float vscale[kReadTokens / 16];
  constexpr int NV = NJ > 1 ? NJ / 2 : 1;
  const int D = c.D, lp = 31 - __builtin_clz(c.P), in_page = c.P - 1;
  const uint32_t per = D / 8, by_per = ((1u << 20) + per - 1) / per, by_d = ((1u << 20) + D - 1) / D;  // x / per = x by_per >> 20
  const int h = blockIdx.x % c.H;
  const int64_t s = blockIdx.x / c.H / windows;
  const int64_t f = first[s] < 0 ? 0 : first[s], e = last[s];
  const int64_t t0 = f / 16 * 16 + (int64_t)(blockIdx.x / c.H % windows) * kReadTokens;
  // Page (times heads) of a token, or of the last one where it is beyond: loads need no branch.
  const int64_t there = (e < width << lp ? e : width << lp) - 1;
  if (there < 0) {
    // nothing held: the rows are zeros (the loads below need one token)
    for (int i = threadIdx.x; i < kReadTokens * (int)per; i += kThreads) {
      const int64_t row = t0 + i / (int)per - f, to = ((s * max_tokens + row) * c.H + h) * D + i % (int)per * 8;
      if (row < 0 || row >= max_tokens) continue;
      if (k_out) *reinterpret_cast<uint4 *>(k_out + to) = make_uint4(0, 0, 0, 0);
      if (v_out) *reinterpret_cast<uint4 *>(v_out + to) = make_uint4(0, 0, 0, 0);
    }
    return;
  }
  auto page_at = [&](int64_t t) {
    const int64_t page = pt[s * width + ((t < there ? t : there) >> lp)];
    return (page < 0 ? 0 : page >= c.pages ? c.pages - 1 : page) * c.H + h;
  };
  int64_t kpage[NJ], vpage[NV];
  int kt[NJ], vg[NV];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    kt[j] = (threadIdx.x + j * kThreads) * by_per >> 20;
    kpage[j] = page_at(t0 + kt[j]);
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    vg[j] = (threadIdx.x + j * kThreads) * by_d >> 20;
    vpage[j] = page_at(t0 + 16 * vg[j]);
  }
  uint2 k[NJ];
  float ks[NJ], vs[NV];
  uint4 v[NV];
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int i = threadIdx.x + j * kThreads;
    k[j] = *reinterpret_cast<const uint2 *>(c.kc + ((kpage[j] << lp) + ((t0 + kt[j]) & in_page)) * D + (i - kt[j] * (int)per) * 8);
    ks[j] = c.ks[kpage[j]];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = threadIdx.x + j * kThreads;
    v[j] = *reinterpret_cast<const uint4 *>(c.vc + ((vpage[j] << lp) + ((t0 + 16 * vg[j]) & in_page)) * D + (i - vg[j] * D) * 16);
    vs[j] = c.vs[vpage[j]];
  }
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int i = threadIdx.x + j * kThreads, ch = i - vg[j] * D;
    if (vg[j] >= kReadTokens / 16) continue;
    *reinterpret_cast<uint4 *>(vt + vg[j] * 18 * D + (ch + ch / 8) * 16) = v[j];
    if (ch == 0) vscale[vg[j]] = vs[j];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < NJ; ++j) {
    const int i = threadIdx.x + j * kThreads, t = kt[j], piece = i - t * (int)per;
    const int64_t row = t0 + t - f;
    if (t >= kReadTokens || row < 0 || row >= max_tokens) continue;
    const bool on = t0 + t <= there;
    const int64_t to = ((s * max_tokens + row) * c.H + h) * D + piece * 8;
    float x[8];
    if (k_out) {
#pragma unroll
      for (int b = 0; b < 8; ++b) x[b] = on ? (float)(int8_t)((b < 4 ? k[j].x : k[j].y) >> (8 * (b % 4))) * ks[j] : 0.0f;
      *reinterpret_cast<uint4 *>(k_out + to) = pack8(x);
    }
    if (v_out) {
      const int8_t *at = reinterpret_cast<const int8_t *>(vt + t / 16 * 18 * D + piece * 144 + t % 16);
#pragma unroll
      for (int b = 0; b < 8; ++b) x[b] = on ? (float)at[16 * b] * vscale[t / 16] : 0.0f;
      *reinterpret_cast<uint4 *>(v_out + to) = pack8(x);
    }
  }
}

// Heads of a token that one lane group takes in turn, with the token's angles and the weights in
// registers: up to `most`, where there are groups enough to fill the card (eight waves a SIMD).
int slices(int64_t tokens, int H, int L, int most) {
  if (H == 0) return 0;
  int per = most;
  while (per > 1 && tokens * ((H + per - 1) / per) * L / 64 < 8192) per /= 2;
  return (H + per - 1) / per;
}

int lanes_of(int D) {
  int L = 1;
  while (L < D / 16) L *= 2;
  return L;
}

template <typename F>
hipError_t with_lanes(int D, F f) {
  switch (lanes_of(D)) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 4: return f(std::integral_constant<int, 4>{});
    case 8: return f(std::integral_constant<int, 8>{});
    default: return f(std::integral_constant<int, 16>{});
  }
}

}  // namespace

hipError_t launch_rope_table(const double *inv_freq, double magnitude, int64_t length, int64_t pairs, float2 *table,
                             hipStream_t s) {
  rope_table_kernel<<<dim3((unsigned)((length * pairs + 255) / 256)), 256, 0, s>>>(inv_freq, magnitude, length, pairs,
                                                                                 table);
  return hipGetLastError();
}

hipError_t launch_qk_rope(const Heads &q, int Hq, const Heads &k, int Hk, const Rope &r, int64_t T, int D,
                          uint16_t *q_out, uint16_t *k_out, hipStream_t s) {
  return with_lanes(D, [&](auto l) {
    constexpr int L = decltype(l)::value;
    const int64_t blocks = (T * (Hq + Hk) + kThreads / L - 1) / (kThreads / L);
    qk_rope_kernel<L><<<dim3((unsigned)blocks), kThreads, 0, s>>>(q, Hq, k, Hk, r, T, D, q_out, k_out);
    return hipGetLastError();
  });
}

hipError_t launch_cache_append(const Cache &c, const Batch &b, const Heads &k, const Heads &v, const Heads &q, int Hq,
                               const Rope &r, int64_t T, uint16_t *q_out, hipStream_t s) {
  return with_lanes(c.D, [&](auto l) {
    constexpr int L = decltype(l)::value;
    const int pages = (int)((b.max_new + 2 * c.P - 2) / c.P);  // pages that max_new tokens can reach
    const int64_t kv_items = b.seqs * pages * c.H * 2;
    const int Sq = slices(b.seqs * b.max_new, Hq, L, 8);
    const int64_t q_blocks = Hq ? (b.max_new * Sq + kThreads / L - 1) / (kThreads / L) : 0;
    const unsigned blocks = (unsigned)(kv_items + b.seqs * q_blocks);
    const size_t lds = (size_t)c.P * c.D / 16 * 17;
    const int64_t tokens = b.max_new < c.P ? b.max_new : c.P;  // of a page
    auto go = [&](auto np) {
      cache_append_kernel<L, decltype(np)::value><<<dim3(blocks), kThreads, lds, s>>>(c, b, k, v, q, Hq, Sq, kv_items, pages,
                                                                                   q_blocks, r, T, q_out);
      return hipGetLastError();
    };
    const int64_t passes = (tokens + kThreads / L - 1) / (kThreads / L);
    if (passes <= 1) return go(std::integral_constant<int, 1>{});
    if (passes <= 2) return go(std::integral_constant<int, 2>{});
    if (passes <= 4) return go(std::integral_constant<int, 4>{});
    return go(std::integral_constant<int, 8>{});
  });
}

hipError_t launch_cache_read(const Cache &c, const int32_t *pt, int64_t width, const int32_t *first,
                             const int32_t *last, int64_t seqs, int64_t max_tokens, uint16_t *k_out, uint16_t *v_out,
                             hipStream_t s) {
  const int windows = (int)((max_tokens + 15 + kReadTokens - 1) / kReadTokens);
  const dim3 grid((unsigned)(seqs * windows * c.H));
  if (c.D <= 32)
    cache_read_kernel<1><<<grid, kThreads, 0, s>>>(c, pt, width, first, last, windows, max_tokens, k_out, v_out);
  else if (c.D <= 64)
    cache_read_kernel<2><<<grid, kThreads, 0, s>>>(c, pt, width, first, last, windows, max_tokens, k_out, v_out);
  else if (c.D <= 128)
    cache_read_kernel<4><<<grid, kThreads, 0, s>>>(c, pt, width, first, last, windows, max_tokens, k_out, v_out);
  else
    cache_read_kernel<8><<<grid, kThreads, 0, s>>>(c, pt, width, first, last, windows, max_tokens, k_out, v_out);
  return hipGetLastError();
}

}  // namespace fq
