// Launchers of the attention operators (internal to libfq) and their argument blocks.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace fq {

// bf16 rows of heads, strides in elements.
struct Heads {
  const uint16_t *p;
  int64_t bs, ts, hs;
};

struct Rope {
  const float2 *table;  // [length][rot / 2] (cos, sin), or NULL
  int64_t length;
  const int32_t *positions;
  const float *qw, *kw;
  float eps;
  int rot, interleaved;
};

struct Cache {
  int8_t *kc;
  float *ks;
  int8_t *vc;
  float *vs;
  int64_t pages;
  int H, P, D;
  float growth;  // of a scale that has to grow, at least
};

struct Batch {
  const int32_t *q_start, *kv_len, *pt;
  int64_t width, seqs, max_new, max_kv;
};

hipError_t launch_rope_table(const double *inv_freq, double magnitude, int64_t length, int64_t pairs, float2 *table,
                             hipStream_t s);
hipError_t launch_qk_rope(const Heads &q, int Hq, const Heads &k, int Hk, const Rope &r, int64_t T, int D,
                          uint16_t *q_out, uint16_t *k_out, hipStream_t s);
hipError_t launch_cache_append(const Cache &c, const Batch &b, const Heads &k, const Heads &v, const Heads &q, int Hq,
                               const Rope &r, int64_t T, uint16_t *q_out, hipStream_t s);
hipError_t launch_cache_read(const Cache &c, const int32_t *pt, int64_t width, const int32_t *first,
                             const int32_t *last, int64_t seqs, int64_t max_tokens, uint16_t *k_out, uint16_t *v_out,
                             hipStream_t s);

// Attention over either source of keys and values.
struct AttnArgs {
  Heads q;
  int Hq, Hk, D;
  int64_t T;         // rows of q and out (ragged batch)
  uint16_t *out;
  float scale;
  int causal;
  int64_t seqs, max_new, max_kv;
  // 8-bit cache
  Cache c;
  Batch b;
  // bf16 states
  Heads k, v;
  const int32_t *kv_len;
  const uint8_t *mask;
  int64_t mask_stride;
};
size_t attention_workspace(bool cached, int Hq, int Hk, int D, int64_t seqs, int64_t max_new, int64_t max_kv);
hipError_t launch_attention(bool cached, const AttnArgs &a, void *ws, hipStream_t s);

}  // namespace fq
