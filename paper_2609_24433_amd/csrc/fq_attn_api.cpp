// C ABI of the attention operators: argument validation and dispatch.  Every check runs before
// anything is enqueued, so a failing call has no device effect.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/fq.h"
#include "fq_attn.hpp"
#include "fq_status.hpp"

namespace {

using namespace fq;

constexpr int64_t kMaxTokens = 1ll << 24;  // rows, sequences and table entries a call
constexpr int64_t kMaxLength = 1ll << 30;  // tokens of a sequence in the cache
constexpr int kMaxHeads = 1024;

// Index arrays are read element by element.
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

fq_status check_head(int D) {
  if (D < 16 || D > 256 || D % 16) return fail(FQ_ERR_UNSUPPORTED, "head size %d is not a multiple of 16 in [16, 256]", D);
  return FQ_OK;
}

fq_status check_groups(int Hq, int Hk) {
  if (Hq < 1 || Hk < 1 || Hq > kMaxHeads) return fail(FQ_ERR_SHAPE, "Hq=%d, Hk=%d: outside [1, %d]", Hq, Hk, kMaxHeads);
  if (Hq % Hk) return fail(FQ_ERR_SHAPE, "Hq=%d is not a multiple of Hk=%d", Hq, Hk);
  return FQ_OK;
}

fq_status check_count(const char *what, int64_t n, int64_t most) {
  if (n < 0) return fail(FQ_ERR_SHAPE, "%s=%lld < 0", what, (long long)n);
  if (n > most) return fail(FQ_ERR_UNSUPPORTED, "%s=%lld: at most %lld", what, (long long)n, (long long)most);
  return FQ_OK;
}

// A view of rows [B][S][H][D]; strides of counts of 1 are not looked at (and set to 0).
fq_status check_heads(const char *what, const fq_heads *x, int64_t B, int64_t S, int64_t H, int D, Heads *out) {
  if (!x || !x->p) return fail(FQ_ERR_NULL, "%s must be non-NULL", what);
  if (!aligned16(x->p)) return fail(FQ_ERR_ALIGN, "%s must be 16-byte aligned", what);
  Heads h;
  h.p = static_cast<const uint16_t *>(x->p);
  h.bs = B > 1 ? x->batch_stride : 0;
  h.ts = S > 1 ? x->token_stride : 0;
  h.hs = H > 1 ? x->head_stride : 0;
  if (h.bs < 0 || h.ts < 0 || h.hs < 0) return fail(FQ_ERR_SHAPE, "%s: a stride is negative", what);
  if (h.bs % 8 || h.ts % 8 || h.hs % 8) return fail(FQ_ERR_ALIGN, "%s: strides must be multiples of 8", what);
  if (h.bs > (1ll << 40) || h.ts > (1ll << 24) || h.hs > (1ll << 32))
    return fail(FQ_ERR_UNSUPPORTED, "%s: a stride is too large", what);
  *out = h;
  return FQ_OK;
}

// Bytes from the first to past the last element of a view.
Span heads_span(const Heads &x, int64_t B, int64_t S, int64_t H, int D) {
  if (!x.p || B <= 0 || S <= 0 || H <= 0) return Span{0, 0};
  return span(x.p, (size_t)((B - 1) * x.bs + (S - 1) * x.ts + (H - 1) * x.hs + D) * 2);
}

fq_status check_rope(const fq_head_rope *r, int D, Rope *out) {
  Rope o{};
  if (r) {
    if (r->rot < 0 || r->rot > D) return fail(FQ_ERR_SHAPE, "rotary part %d outside [0, %d]", r->rot, D);
    if (r->rot % 16) return fail(FQ_ERR_UNSUPPORTED, "rotary part %d is not a multiple of 16", r->rot);
    if (r->rot > 0) {
      if (!r->table) return fail(FQ_ERR_NULL, "a rotation needs its table");
      if (r->length < 1 || r->length > kMaxLength) return fail(FQ_ERR_SHAPE, "table length %lld", (long long)r->length);
    }
    if (!(r->eps >= 0.0f) || std::isinf(r->eps)) return fail(FQ_ERR_UNSUPPORTED, "eps=%g", (double)r->eps);
    if ((r->table && !aligned16(r->table)) || (r->q_weight && !aligned16(r->q_weight)) ||
        (r->k_weight && !aligned16(r->k_weight)) || !aligned4(r->positions))
      return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned, index arrays 4-byte");
    o.table = reinterpret_cast<const float2 *>(r->table);
    o.length = r->length;
    o.positions = r->positions;
    o.qw = r->q_weight;
    o.kw = r->k_weight;
    o.eps = r->eps;
    o.rot = r->rot;
    o.interleaved = r->interleaved != 0;
  }
  *out = o;
  return FQ_OK;
}

struct RopeSpans {
  Span table, positions, qw, kw;
};
RopeSpans rope_spans(const Rope &r, int64_t T, int D) {
  return RopeSpans{span(r.rot ? r.table : nullptr, (size_t)r.length * r.rot * 4), span(r.positions, (size_t)T * 4),
                   span(r.qw, (size_t)D * 4), span(r.kw, (size_t)D * 4)};
}

fq_status check_cache(const fq_kv_cache *c, Cache *out) {
  if (!c) return fail(FQ_ERR_NULL, "the cache must be non-NULL");
  fq_status s;
  if ((s = check_head(c->head_dim)) != FQ_OK) return s;
  const int P = c->page_tokens;
  if (P != 16 && P != 32 && P != 64 && P != 128)
    return fail(FQ_ERR_UNSUPPORTED, "pages of %d tokens (must be 16, 32, 64 or 128)", P);
  if (c->heads < 1 || c->heads > kMaxHeads) return fail(FQ_ERR_SHAPE, "%d cache heads outside [1, %d]", c->heads, kMaxHeads);
  if (c->pages < 1 || c->pages > 0x7FFFFFFFll) return fail(FQ_ERR_SHAPE, "%lld cache pages", (long long)c->pages);
  if (!c->k_codes || !c->k_scale || !c->v_codes || !c->v_scale)
    return fail(FQ_ERR_NULL, "the cache's codes and scales must be non-NULL");
  if (!aligned16(c->k_codes) || !aligned16(c->k_scale) || !aligned16(c->v_codes) || !aligned16(c->v_scale))
    return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned");
  *out = Cache{static_cast<int8_t *>(c->k_codes), c->k_scale, static_cast<int8_t *>(c->v_codes), c->v_scale, c->pages,
               c->heads, P, c->head_dim, 1.0f};
  return FQ_OK;
}

struct CacheSpans {
  Span kc, ks, vc, vs;
};
CacheSpans cache_spans(const Cache &c) {
  const size_t rows = (size_t)c.pages * c.H;
  return CacheSpans{span(c.kc, rows * c.P * c.D), span(c.ks, rows * 4), span(c.vc, rows * c.P * c.D),
                    span(c.vs, rows * 4)};
}

fq_status check_batch(const fq_kv_batch *b, const Cache &c, Batch *out) {
  if (!b) return fail(FQ_ERR_NULL, "the batch must be non-NULL");
  fq_status s;
  if ((s = check_count("seqs", b->seqs, 65535)) != FQ_OK) return s;
  if ((s = check_count("max_new", b->max_new, kMaxTokens)) != FQ_OK) return s;
  if ((s = check_count("max_kv", b->max_kv, kMaxLength)) != FQ_OK) return s;
  if ((s = check_count("table_width", b->table_width, kMaxTokens * 8)) != FQ_OK) return s;
  if (b->table_width * c.P < b->max_kv)
    return fail(FQ_ERR_SHAPE, "a table of %lld pages does not hold max_kv=%lld tokens", (long long)b->table_width,
                (long long)b->max_kv);
  if (b->seqs > 0 && (!b->q_start || !b->kv_len || (b->max_kv > 0 && !b->page_table)))
    return fail(FQ_ERR_NULL, "q_start, kv_len and page_table must be non-NULL");
  if (!aligned4(b->q_start) || !aligned4(b->kv_len) || !aligned4(b->page_table))
    return fail(FQ_ERR_ALIGN, "index arrays must be 4-byte aligned");
  *out = Batch{b->q_start, b->kv_len, b->page_table, b->table_width, b->seqs, b->max_new, b->max_kv};
  return FQ_OK;
}

// The outputs against each other and the inputs, with the batch's arrays among the inputs.
bool batch_alias(std::initializer_list<Span> outs, std::initializer_list<Span> ins, const Batch &b) {
  return outputs_alias(outs, ins) ||
         outputs_alias(outs, {span(b.q_start, (size_t)(b.seqs + 1) * 4), span(b.kv_len, (size_t)b.seqs * 4),
                              span(b.pt, (size_t)b.seqs * b.width * 4)});
}

fq_status check_ws(const void *ws, size_t have, size_t need) {
  if (need > 0 && (!ws || have < need))
    return fail(FQ_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws ? have : (size_t)0);
  if (need > 0 && !aligned16(ws)) return fail(FQ_ERR_ALIGN, "workspace must be 16-byte aligned");
  return FQ_OK;
}

fq_status check_scale(float scale) {
  if (!(scale > 0.0f) || std::isinf(scale)) return fail(FQ_ERR_UNSUPPORTED, "scale=%g (must be positive)", (double)scale);
  return FQ_OK;
}

// Workgroups of a launch stay within 31 bits.
fq_status check_grid(double blocks) {
  if (blocks > 2147483647.0) return fail(FQ_ERR_UNSUPPORTED, "the call needs %.0f workgroups", blocks);
  return FQ_OK;
}

}  // namespace

extern "C" {

fq_status fq_rope_table(const double *inv_freq, double magnitude, int64_t length, int64_t pairs, float *table,
                        void *stream) {
  fq_status s;
  if ((s = check_count("length", length, kMaxLength)) != FQ_OK) return s;
  if ((s = check_count("pairs", pairs, 128)) != FQ_OK) return s;
  if ((s = check_grid((double)length * (double)pairs / 256 + 1)) != FQ_OK) return s;
  if (length == 0 || pairs == 0) return ok();
  if (!inv_freq || !table) return fail(FQ_ERR_NULL, "inv_freq and table must be non-NULL");
  if (!aligned16(inv_freq) || !aligned16(table)) return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned");
  if (overlap(span(table, (size_t)length * pairs * 8), span(inv_freq, (size_t)pairs * 8)))
    return fail(FQ_ERR_ALIAS, "table must not overlap inv_freq");
  hipError_t e = launch_rope_table(inv_freq, magnitude, length, pairs, reinterpret_cast<float2 *>(table),
                                   static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "rope_table launch");
  return ok();
}

fq_status fq_qk_rope(const fq_heads *q, int Hq, const fq_heads *k, int Hk, const fq_head_rope *rope, int64_t T, int D,
                     void *q_out, void *k_out, void *stream) {
  fq_status s;
  Rope r;
  Heads hq{}, hk{};
  if ((s = check_head(D)) != FQ_OK) return s;
  if ((s = check_count("T", T, kMaxTokens)) != FQ_OK) return s;
  if ((s = check_count("Hq", Hq, kMaxHeads)) != FQ_OK) return s;
  if ((s = check_count("Hk", Hk, kMaxHeads)) != FQ_OK) return s;
  if (!rope) return fail(FQ_ERR_NULL, "rope must be non-NULL");
  if ((s = check_rope(rope, D, &r)) != FQ_OK) return s;
  if (T == 0 || Hq + Hk == 0) return ok();
  if (Hq && (s = check_heads("q", q, 1, T, Hq, D, &hq)) != FQ_OK) return s;
  if (Hk && (s = check_heads("k", k, 1, T, Hk, D, &hk)) != FQ_OK) return s;
  if ((Hq && !q_out) || (Hk && !k_out)) return fail(FQ_ERR_NULL, "q_out and k_out must be non-NULL");
  if ((Hq && !aligned16(q_out)) || (Hk && !aligned16(k_out))) return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned");
  const RopeSpans rs = rope_spans(r, T, D);
  if (outputs_alias({span(Hq ? q_out : nullptr, (size_t)T * Hq * D * 2), span(Hk ? k_out : nullptr, (size_t)T * Hk * D * 2)},
                    {heads_span(hq, 1, T, Hq, D), heads_span(hk, 1, T, Hk, D), rs.table, rs.positions, rs.qw, rs.kw}))
    return fail(FQ_ERR_ALIAS, "q_out and k_out must not overlap each other or an input");
  hipError_t e = launch_qk_rope(hq, Hq, hk, Hk, r, T, D, static_cast<uint16_t *>(q_out), static_cast<uint16_t *>(k_out),
                                static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "qk_rope launch");
  return ok();
}

fq_status fq_cache_append(const fq_kv_cache *cache, const fq_kv_batch *batch, const fq_heads *k, const fq_heads *v,
                          const fq_heads *q, int Hq, const fq_head_rope *rope, int64_t T, void *q_out, void *stream) {
  fq_status s;
  Cache c;
  Batch b;
  Rope r;
  Heads hk, hv, hq{};
  if ((s = check_cache(cache, &c)) != FQ_OK) return s;
  if (cache->growth < 0 || cache->growth > 100) return fail(FQ_ERR_UNSUPPORTED, "growth=%d outside [0, 100]", cache->growth);
  c.growth = 1.0f + (float)cache->growth / 100.0f;
  if ((s = check_batch(batch, c, &b)) != FQ_OK) return s;
  if ((s = check_count("T", T, kMaxTokens)) != FQ_OK) return s;
  if ((s = check_count("Hq", Hq, kMaxHeads)) != FQ_OK) return s;
  if ((s = check_rope(rope, c.D, &r)) != FQ_OK) return s;
  if ((s = check_grid((double)b.seqs * ((double)(b.max_new / c.P + 2) * c.H * 2 + ((double)b.max_new * Hq / 16 + 1)))) != FQ_OK)
    return s;
  if (T == 0 || b.seqs == 0 || b.max_new == 0 || (b.max_kv == 0 && Hq == 0)) return ok();
  if ((s = check_heads("k", k, 1, T, c.H, c.D, &hk)) != FQ_OK) return s;
  if ((s = check_heads("v", v, 1, T, c.H, c.D, &hv)) != FQ_OK) return s;
  if (Hq) {
    if ((s = check_heads("q", q, 1, T, Hq, c.D, &hq)) != FQ_OK) return s;
    if (!q_out) return fail(FQ_ERR_NULL, "q_out must be non-NULL");
    if (!aligned16(q_out)) return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned");
  }
  const CacheSpans cs = cache_spans(c);
  const RopeSpans rs = rope_spans(r, T, c.D);
  if (batch_alias({cs.kc, cs.ks, cs.vc, cs.vs, span(Hq ? q_out : nullptr, (size_t)T * Hq * c.D * 2)},
                  {heads_span(hk, 1, T, c.H, c.D), heads_span(hv, 1, T, c.H, c.D), heads_span(hq, 1, T, Hq, c.D), rs.table,
                   rs.positions, rs.qw, rs.kw},
                  b))
    return fail(FQ_ERR_ALIAS, "the cache and q_out must not overlap each other or an input");
  hipError_t e = launch_cache_append(c, b, hk, hv, hq, Hq, r, T, static_cast<uint16_t *>(q_out),
                                     static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "cache_append launch");
  return ok();
}

fq_status fq_cache_read(const fq_kv_cache *cache, const int32_t *page_table, int64_t table_width,
                        const int32_t *first, const int32_t *last, int64_t seqs, int64_t max_tokens, void *k_out,
                        void *v_out, void *stream) {
  fq_status s;
  Cache c;
  if ((s = check_cache(cache, &c)) != FQ_OK) return s;
  if ((s = check_count("seqs", seqs, 65535)) != FQ_OK) return s;
  if ((s = check_count("table_width", table_width, kMaxTokens * 8)) != FQ_OK) return s;
  if ((s = check_count("max_tokens", max_tokens, kMaxLength)) != FQ_OK) return s;
  if ((s = check_grid((double)seqs * (double)(max_tokens / 16 + 2) * c.H)) != FQ_OK) return s;
  if (seqs == 0 || max_tokens == 0 || (!k_out && !v_out)) return ok();
  if (!first || !last || (table_width > 0 && !page_table))
    return fail(FQ_ERR_NULL, "page_table, first and last must be non-NULL");
  if (!aligned4(page_table) || !aligned4(first) || !aligned4(last) || !aligned16(k_out) || !aligned16(v_out))
    return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned, index arrays 4-byte");
  const CacheSpans cs = cache_spans(c);
  const size_t n = (size_t)seqs * max_tokens * c.H * c.D * 2;
  if (outputs_alias({span(k_out, k_out ? n : 0), span(v_out, v_out ? n : 0)},
                    {cs.kc, cs.ks, cs.vc, cs.vs, span(page_table, (size_t)seqs * table_width * 4),
                     span(first, (size_t)seqs * 4), span(last, (size_t)seqs * 4)}))
    return fail(FQ_ERR_ALIAS, "k_out and v_out must not overlap each other or an input");
  hipError_t e = launch_cache_read(c, page_table, table_width, first, last, seqs, max_tokens,
                                   static_cast<uint16_t *>(k_out), static_cast<uint16_t *>(v_out),
                                   static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "cache_read launch");
  return ok();
}

size_t fq_cache_attention_workspace_bytes(int64_t T, int Hq, int Hk, int D, int64_t seqs, int64_t max_new,
                                          int64_t max_kv) {
  if (T <= 0 || Hq < 1 || Hk < 1 || Hq % Hk || D < 16 || D > 256 || D % 16 || seqs <= 0 || max_new <= 0 || max_kv <= 0)
    return 0;
  return attention_workspace(true, Hq, Hk, D, seqs, max_new, max_kv);
}

fq_status fq_cache_attention(const fq_heads *q, int Hq, int64_t T, const fq_kv_cache *cache, const fq_kv_batch *batch,
                             float scale, int causal, void *out, void *ws, size_t ws_bytes, void *stream) {
  fq_status s;
  AttnArgs a{};
  if ((s = check_cache(cache, &a.c)) != FQ_OK) return s;
  if ((s = check_batch(batch, a.c, &a.b)) != FQ_OK) return s;
  if ((s = check_groups(Hq, a.c.H)) != FQ_OK) return s;
  if ((s = check_count("T", T, kMaxTokens)) != FQ_OK) return s;
  if ((s = check_scale(scale)) != FQ_OK) return s;
  if ((s = check_grid((double)a.b.max_new * Hq)) != FQ_OK) return s;
  if (T == 0 || a.b.seqs == 0 || a.b.max_new == 0) return ok();
  if ((s = check_heads("q", q, 1, T, Hq, a.c.D, &a.q)) != FQ_OK) return s;
  if (!out) return fail(FQ_ERR_NULL, "out must be non-NULL");
  if (!aligned16(out)) return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned");
  const size_t need = fq_cache_attention_workspace_bytes(T, Hq, a.c.H, a.c.D, a.b.seqs, a.b.max_new, a.b.max_kv);
  if ((s = check_ws(ws, ws_bytes, need)) != FQ_OK) return s;
  const CacheSpans cs = cache_spans(a.c);
  if (batch_alias({span(out, (size_t)T * Hq * a.c.D * 2), span(need ? ws : nullptr, need)},
                  {heads_span(a.q, 1, T, Hq, a.c.D), cs.kc, cs.ks, cs.vc, cs.vs}, a.b))
    return fail(FQ_ERR_ALIAS, "out and the workspace must not overlap each other or an input");
  a.Hq = Hq;
  a.Hk = a.c.H;
  a.D = a.c.D;
  a.T = T;
  a.out = static_cast<uint16_t *>(out);
  a.scale = scale;
  a.causal = causal != 0;
  a.seqs = a.b.seqs;
  a.max_new = a.b.max_new;
  a.max_kv = a.b.max_kv;
  hipError_t e = launch_attention(true, a, ws, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "cache_attention launch");
  return ok();
}

size_t fq_cross_attention_workspace_bytes(int64_t B, int64_t Sq, int64_t Sk, int Hq, int Hk, int D) {
  if (B <= 0 || Sq <= 0 || Sk <= 0 || Hq < 1 || Hk < 1 || Hq % Hk || D < 16 || D > 256 || D % 16) return 0;
  return attention_workspace(false, Hq, Hk, D, B, Sq, Sk);
}

fq_status fq_cross_attention(const fq_heads *q, const fq_heads *k, const fq_heads *v, const int32_t *kv_len,
                             const uint8_t *key_mask, int64_t mask_stride, int64_t B, int64_t Sq, int64_t Sk, int Hq,
                             int Hk, int D, float scale, void *out, void *ws, size_t ws_bytes, void *stream) {
  fq_status s;
  AttnArgs a{};
  if ((s = check_head(D)) != FQ_OK) return s;
  if ((s = check_groups(Hq, Hk)) != FQ_OK) return s;
  if ((s = check_count("B", B, 65535)) != FQ_OK) return s;
  if ((s = check_count("Sq", Sq, kMaxTokens)) != FQ_OK) return s;
  if ((s = check_count("Sk", Sk, kMaxTokens)) != FQ_OK) return s;
  if ((s = check_scale(scale)) != FQ_OK) return s;
  if ((s = check_grid((double)Sq * Hq)) != FQ_OK) return s;
  if (key_mask && (mask_stride < 0 || mask_stride > (1ll << 40)))
    return fail(FQ_ERR_SHAPE, "mask_stride=%lld", (long long)mask_stride);
  if (B == 0 || Sq == 0) return ok();
  if ((s = check_heads("q", q, B, Sq, Hq, D, &a.q)) != FQ_OK) return s;
  if (Sk > 0) {
    if ((s = check_heads("k", k, B, Sk, Hk, D, &a.k)) != FQ_OK) return s;
    if ((s = check_heads("v", v, B, Sk, Hk, D, &a.v)) != FQ_OK) return s;
  }
  if (!out) return fail(FQ_ERR_NULL, "out must be non-NULL");
  if (!aligned16(out) || !aligned4(kv_len)) return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned, index arrays 4-byte");
  const size_t need = fq_cross_attention_workspace_bytes(B, Sq, Sk, Hq, Hk, D);
  if ((s = check_ws(ws, ws_bytes, need)) != FQ_OK) return s;
  if (outputs_alias({span(out, (size_t)B * Sq * Hq * D * 2), span(need ? ws : nullptr, need)},
                    {heads_span(a.q, B, Sq, Hq, D), heads_span(a.k, B, Sk, Hk, D), heads_span(a.v, B, Sk, Hk, D),
                     span(kv_len, (size_t)B * 4), span(key_mask, (size_t)((B - 1) * mask_stride + Sk))}))
    return fail(FQ_ERR_ALIAS, "out and the workspace must not overlap each other or an input");
  a.Hq = Hq;
  a.Hk = Hk;
  a.D = D;
  a.T = B * Sq;
  a.out = static_cast<uint16_t *>(out);
  a.scale = scale;
  a.seqs = B;
  a.max_new = Sq;
  a.max_kv = Sk;
  a.kv_len = kv_len;
  a.mask = key_mask;
  a.mask_stride = mask_stride;
  hipError_t e = launch_attention(false, a, ws, static_cast<hipStream_t>(stream));
  if (e != hipSuccess) return hip_fail(e, "cross_attention launch");
  return ok();
}

}  // extern "C"
