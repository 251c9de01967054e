// Norms of queries and keys per head, the position rotation, and appends to the 8-bit cache.
//
// A head of D values is held by D/16 lanes of a group of L (the next power of two), 16 values a
// lane: the two 8-value chunks that the rotation pairs, dims [8m, 8m + 8) and the same R/2
// further on (halves), or 16 adjacent dims (adjacent pairs, and dims the rotation leaves alone).
// So a rotation never crosses lanes, and the only exchange is the norm's sum.
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

__device__ __forceinline__ void load_head(const uint16_t *x, const Place &p, float (&v)[16]) {
  uint4 u0 = make_uint4(0, 0, 0, 0), u1 = u0;
  if (p.in) {
    u0 = *reinterpret_cast<const uint4 *>(x + p.a);
    u1 = *reinterpret_cast<const uint4 *>(x + p.b);
  }
  unpack8(u0, v);
  unpack8(u1, v + 8);
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

// One token's heads slice, slice + S, ... of H: its angles and weights stay in registers.
template <int L>
__device__ __forceinline__ void rope_heads(const uint16_t *x, int64_t hs, uint16_t *y, int H, int slice, int S,
                                           const Rope &r, const float *w, const Place &p, const float2 (&cs)[8], int D) {
  float g[16];
  load_weight(w, p, g);
  for (int h = slice; h < H; h += S) {
    float v[16];
    load_head(x + h * hs, p, v);
    norm_rotate<L>(v, w != nullptr, g, cs, p, r.interleaved, r.eps, D);
    store_head(y + (int64_t)h * D, p, v);
  }
}

// Grid: units of (token, slice); a token has Sq slices of query heads, then Sk of key heads.
template <int L>
__global__ __launch_bounds__(kThreads) void qk_rope_kernel(Heads q, int Hq, int Sq, Heads k, int Hk, int Sk, Rope r,
                                                           int64_t T, int D, uint16_t *__restrict__ q_out,
                                                           uint16_t *__restrict__ k_out) {
  const int64_t u = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
  const int S = Sq + Sk, m = threadIdx.x % L;
  const int64_t t = u / S;
  if (t >= T) return;
  const int slice = (int)(u - t * S);
  const Place p = place_of(m, D, r.rot, r.interleaved);
  float2 cs[8];
  load_angles(r, p, m, r.positions ? r.positions[t] : t, cs);
  if (slice < Sq)
    rope_heads<L>(q.p + t * q.ts, q.hs, q_out + t * Hq * D, Hq, slice, Sq, r, r.qw, p, cs, D);
  else
    rope_heads<L>(k.p + t * k.ts, k.hs, k_out + t * Hk * D, Hk, slice - Sq, Sk, r, r.kw, p, cs, D);
}

// ---------------------------------------------------------------- appends

// The rows of sequence s in this call: [row, row + n), and the slot of its first token (which may
// be negative where kv_len is short: those tokens are dropped).
struct Span1 {
  int64_t row;
  int n;
  int64_t begin, end;  // slots
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
  r.begin = m - n;
  r.end = m < b.max_kv ? m : b.max_kv;
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

// Workgroups [0, kv_items): one page of one sequence and head, keys or values; all of the page's
// new tokens are read twice (the second time from a cache) for the scale and then the codes.
// The others: the query heads of the new tokens.
template <int L>
__global__ __launch_bounds__(kThreads) void cache_append_kernel(Cache c, Batch b, Heads k, Heads v, Heads q, int Hq,
                                                                int Sq, int64_t kv_items, int pages_per_seq,
                                                                int64_t q_blocks, Rope r, int64_t T,
                                                                uint16_t *__restrict__ q_out) {
  extern __shared__ __align__(16) uint8_t tile[];  // values: the page's new codes, [P/16][D][16]
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
  const int held = (int)(first > lo ? first - lo : 0);
  const int64_t page = page_of(b, c.pages, s, pw) * c.H + h;
  const Place pl = keys ? p : place_of(m, D, 0, 0);
  float g[16];
  load_weight(keys ? r.kw : nullptr, pl, g);

  auto token = [&](int64_t slot, float(&x)[16]) {
    const int64_t t = sp.row + (slot - sp.begin);
    if (keys) {
      float2 cs[8];
      load_angles(r, pl, m, r.positions ? r.positions[t] : slot, cs);
      load_head(k.p + t * k.ts + h * k.hs, pl, x);
      norm_rotate<L>(x, r.kw != nullptr, g, cs, pl, r.interleaved, r.eps, D);
    } else {
      load_head(v.p + t * v.ts + h * v.hs, pl, x);
    }
  };

  uint32_t top = 0;
  for (int64_t slot = s0 + grp; slot < s1; slot += NG) {
    float x[16];
    token(slot, x);
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t a = abs_bits(x[i]);
      top = a > top ? a : top;
    }
  }
  top = block_max(top, red);
  float *scale_at = (keys ? c.ks : c.vs) + page;
  const float old = held ? *scale_at : 0.0f;
  float scale = __uint_as_float(top) / 127.0f;
  bool bad = top >= 0x7F800000u;
  if (held) {
    bad = bad || old != old;
    scale = old > scale ? old : scale;
  }
  if (!(scale >= FLT_MIN)) scale = 0.0f;
  const bool grew = held && !bad && scale != old;
  const float inv = scale > 0.0f && !bad ? 1.0f / scale : 0.0f;
  const float ratio = scale > 0.0f ? old / scale : 0.0f;
  __syncthreads();  // every thread has read the old scale
  if (threadIdx.x == 0) *scale_at = bad ? __uint_as_float(0x7FC00000u) : scale;

  if (keys) {
    int8_t *base = c.kc + page * P * D;
    if (grew)
      for (int i = threadIdx.x; i < held * D / 16; i += kThreads) {
        uint4 *w = reinterpret_cast<uint4 *>(base) + i;
        const uint4 o = *w;
        *w = make_uint4(rescale4(o.x, ratio), rescale4(o.y, ratio), rescale4(o.z, ratio), rescale4(o.w, ratio));
      }
    for (int64_t slot = s0 + grp; slot < s1; slot += NG) {
      float x[16];
      token(slot, x);
      uint32_t w[4] = {0, 0, 0, 0};
      if (!bad)
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i / 4] |= ((uint32_t)code_of(x[i], inv) & 0xFFu) << (8 * (i % 4));
      int8_t *row = base + (slot - lo) * D;
      if (pl.in) {
        *reinterpret_cast<uint2 *>(row + pl.a) = make_uint2(w[0], w[1]);
        *reinterpret_cast<uint2 *>(row + pl.b) = make_uint2(w[2], w[3]);
      }
    }
    return;
  }
  for (int64_t slot = s0 + grp; slot < s1; slot += NG) {
    float x[16];
    token(slot, x);
    const int o = (int)(slot - lo);
    uint8_t *to = tile + (o / 16) * D * 16 + o % 16;
    if (pl.in)
#pragma unroll
      for (int i = 0; i < 16; ++i) to[(16 * m + i) * 16] = bad ? 0 : (uint8_t)code_of(x[i], inv);
  }
  __syncthreads();
  // 16 tokens of one channel an item: earlier codes, then the new ones, then zeros
  const int from = (int)(s0 - lo), to = (int)(s1 - lo);
  const int g0 = grew ? 0 : from / 16, g1 = (to + 15) / 16;
  uint4 *base = reinterpret_cast<uint4 *>(c.vc + page * P * D);
  for (int i = g0 * D + threadIdx.x; i < g1 * D; i += kThreads) {
    const int t0 = i / D * 16;
    uint32_t w[4] = {0, 0, 0, 0};
    if (t0 < held) {
      const uint4 o = base[i];
      w[0] = o.x, w[1] = o.y, w[2] = o.z, w[3] = o.w;
      if (grew)
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = rescale4(w[j], ratio);
    }
    const uint4 n = reinterpret_cast<const uint4 *>(tile)[i];
    const uint32_t nw[4] = {n.x, n.y, n.z, n.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int o = t0 + 4 * j + e;
        const uint32_t mask = 0xFFu << (8 * e);
        if (o >= from) w[j] = (w[j] & ~mask) | (o < to ? nw[j] & mask : 0u);
      }
    base[i] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// One 16-token group of one head: codes times scales, the rows of [first, last), zeros beyond.
__global__ __launch_bounds__(kThreads) void cache_read_kernel(Cache c, const int32_t *__restrict__ pt, int64_t width,
                                                              const int32_t *__restrict__ first,
                                                              const int32_t *__restrict__ last, int groups,
                                                              int64_t max_tokens, uint16_t *__restrict__ k_out,
                                                              uint16_t *__restrict__ v_out) {
  __shared__ __align__(16) int8_t vt[256 * 16];
  const int D = c.D, P = c.P;
  const int h = blockIdx.x % c.H;
  const int64_t s = blockIdx.x / c.H / groups;
  const int64_t f = first[s] < 0 ? 0 : first[s], e = last[s];
  const int64_t t0 = (f / 16 + blockIdx.x / c.H % groups) * 16;  // first token of the cache's group
  const int64_t w = t0 / P;
  const bool there = w < width && t0 < e;
  int64_t page = there ? pt[s * width + w] : 0;
  page = (page < 0 ? 0 : page >= c.pages ? c.pages - 1 : page) * c.H + h;
  const int o = (int)(t0 % P);
  const float ks = there ? c.ks[page] : 0.0f, vs = there ? c.vs[page] : 0.0f;
  if (there && v_out)
    for (int i = threadIdx.x; i < D; i += kThreads)
      reinterpret_cast<uint4 *>(vt)[i] = reinterpret_cast<const uint4 *>(c.vc + page * P * D + (int64_t)(o / 16) * D * 16)[i];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * (D / 8); i += kThreads) {
    const int t = i / (D / 8), d = i % (D / 8) * 8;
    const int64_t row = t0 + t - f;
    if (row < 0 || row >= max_tokens) continue;
    const bool on = there && t0 + t < e;
    const int64_t at = ((s * max_tokens + row) * c.H + h) * D + d;
    float x[8];
    if (k_out) {
      uint2 u = make_uint2(0, 0);
      if (on) u = *reinterpret_cast<const uint2 *>(c.kc + page * P * D + (int64_t)(o + t) * D + d);
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = on ? (float)(int8_t)((j < 4 ? u.x : u.y) >> (8 * (j % 4))) * ks : 0.0f;
      *reinterpret_cast<uint4 *>(k_out + at) = pack8(x);
    }
    if (v_out) {
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = on ? (float)vt[(d + j) * 16 + t] * vs : 0.0f;
      *reinterpret_cast<uint4 *>(v_out + at) = pack8(x);
    }
  }
}

// Slices of H heads for `units` tokens: up to 8 heads share a lane group's angles and weights
// where there are groups enough to fill the card (about eight waves a SIMD).
int slices(int64_t tokens, int heads_all, int H, int L) {
  if (H == 0) return 0;
  int per = 8;
  while (per > 1 && tokens * ((heads_all + per - 1) / per) * L / 64 < 8192) per /= 2;
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
    const int Sq = slices(T, Hq + Hk, Hq, L), Sk = slices(T, Hq + Hk, Hk, L);
    const int64_t blocks = (T * (Sq + Sk) + kThreads / L - 1) / (kThreads / L);
    qk_rope_kernel<L><<<dim3((unsigned)blocks), kThreads, 0, s>>>(q, Hq, Sq, k, Hk, Sk, r, T, D, q_out, k_out);
    return hipGetLastError();
  });
}

hipError_t launch_cache_append(const Cache &c, const Batch &b, const Heads &k, const Heads &v, const Heads &q, int Hq,
                               const Rope &r, int64_t T, uint16_t *q_out, hipStream_t s) {
  return with_lanes(c.D, [&](auto l) {
    constexpr int L = decltype(l)::value;
    const int pages = (int)((b.max_new + 2 * c.P - 2) / c.P);  // pages that max_new tokens can reach
    const int64_t kv_items = b.seqs * pages * c.H * 2;
    const int Sq = slices(b.seqs * b.max_new, Hq, Hq, L);
    const int64_t q_blocks = Hq ? (b.max_new * Sq + kThreads / L - 1) / (kThreads / L) : 0;
    cache_append_kernel<L><<<dim3((unsigned)(kv_items + b.seqs * q_blocks)), kThreads, c.P * c.D, s>>>(
        c, b, k, v, q, Hq, Sq, kv_items, pages, q_blocks, r, T, q_out);
    return hipGetLastError();
  });
}

hipError_t launch_cache_read(const Cache &c, const int32_t *pt, int64_t width, const int32_t *first,
                             const int32_t *last, int64_t seqs, int64_t max_tokens, uint16_t *k_out, uint16_t *v_out,
                             hipStream_t s) {
  const int groups = (int)((max_tokens + 15) / 16 + 1);
  cache_read_kernel<<<dim3((unsigned)(seqs * groups * c.H)), kThreads, 0, s>>>(c, pt, width, first, last, groups,
                                                                              max_tokens, k_out, v_out);
  return hipGetLastError();
}

}  // namespace fq
