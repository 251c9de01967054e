// C ABI of the microscaled operators and of the norm before a projection: argument validation and
// dispatch.  Every check runs before anything is enqueued, so a failing call has no device effect.
#include <hip/hip_runtime.h>

#include <cmath>

#include "../../include/fq.h"
#include "fq_launch.hpp"
#include "fq_mx.hpp"
#include "fq_status.hpp"

namespace {

using namespace fq;

constexpr int64_t kMaxK = 32768, kMaxRows = 1ll << 24;

// float nearest to 1/sqrt(b), b a power of two
float root_of(int b) { return (float)(1.0 / std::sqrt((double)b)); }

fq_status check_k(int64_t K) {
  if (K < 128 || K > kMaxK) return fail(FQ_ERR_UNSUPPORTED, "K=%lld outside [128, %lld]", (long long)K, (long long)kMaxK);
  if (K % 128) return fail(FQ_ERR_UNSUPPORTED, "K=%lld is not a multiple of 128", (long long)K);
  return FQ_OK;
}

fq_status check_rows(const char *what, int64_t n) {
  if (n < 0) return fail(FQ_ERR_SHAPE, "%s=%lld < 0", what, (long long)n);
  if (n > kMaxRows) return fail(FQ_ERR_UNSUPPORTED, "%s=%lld: at most %lld", what, (long long)n, (long long)kMaxRows);
  return FQ_OK;
}

fq_status check_block(int b, int64_t K) {
  if (!is_pow2(b) || b > 256) return fail(FQ_ERR_UNSUPPORTED, "b=%d is not a power of two in [1, 256]", b);
  if (K % b) return fail(FQ_ERR_SHAPE, "K=%lld is not a multiple of b=%d", (long long)K, b);
  return FQ_OK;
}

// Row stride of an array of K columns, whose rows stay 16-byte aligned; not looked at for one row.
fq_status check_ld(const char *what, int64_t ld, int64_t K, int mult, int64_t M) {
  if (M <= 1) return FQ_OK;
  if (ld < K) return fail(FQ_ERR_SHAPE, "%s=%lld < %lld columns", what, (long long)ld, (long long)K);
  if (ld % mult) return fail(FQ_ERR_ALIGN, "%s=%lld is not a multiple of %d", what, (long long)ld, mult);
  if (ld > (1ll << 32)) return fail(FQ_ERR_UNSUPPORTED, "%s=%lld is too large", what, (long long)ld);
  return FQ_OK;
}

fq_status check_aligned(std::initializer_list<const void *> ps) {
  for (const void *p : ps)
    if (!aligned16(p)) return fail(FQ_ERR_ALIGN, "pointers must be 16-byte aligned");
  return FQ_OK;
}

size_t mx_codes_bytes(int64_t M, int64_t K) { return (size_t)M * (size_t)K / 2; }
size_t mx_scales_bytes(int64_t M, int64_t K) { return (size_t)M * (size_t)K / 32; }

Span rows_of(const void *p, int64_t M, int64_t ld, int64_t K, int size) {
  return span(p, p ? rows_span(M, ld * size, K * size) : 0);
}
Span floats(const float *p, int64_t n) { return span(p, p ? (size_t)n * 4 : 0); }

#define FQ_TRY(e)                          \
  do {                                     \
    const fq_status s_ = (e);              \
    if (s_ != FQ_OK) return s_;            \
  } while (0)

struct NormCall {
  const void *x;
  int64_t ldx;
  const void *residual;
  int64_t ldr;
  const float *weight;
  float eps;
  const float *post;
  int64_t M, K;
  int b;
  float clip;
  void *sum;
  int64_t lds;
  void *codes, *scales;
  size_t codes_bytes, scales_bytes;
  int fmt;
  void *stream;
};

fq_status norm_common(const NormCall &c) {
  FQ_TRY(check_rows("M", c.M));
  FQ_TRY(check_k(c.K));
  FQ_TRY(check_block(c.b, c.K));
  if (!(c.clip > 0.0f && c.clip <= 1.0f)) return fail(FQ_ERR_UNSUPPORTED, "clip_ratio=%g outside (0, 1]", (double)c.clip);
  if (!(c.eps > 0.0f) || std::isinf(c.eps)) return fail(FQ_ERR_UNSUPPORTED, "eps=%g is not positive and finite", (double)c.eps);
  if (c.sum && !c.residual) return fail(FQ_ERR_NULL, "sum_out needs a residual");
  FQ_TRY(check_ld("ldx", c.ldx, c.K, 8, c.M));
  if (c.residual) FQ_TRY(check_ld("ldr", c.ldr, c.K, 8, c.M));
  if (c.sum) FQ_TRY(check_ld("ld_sum", c.lds, c.K, 8, c.M));
  if (c.M == 0) return ok();
  if (!c.x || !c.weight || !c.codes || !c.scales) return fail(FQ_ERR_NULL, "x, weight, codes and scales must be non-NULL");
  FQ_TRY(check_aligned({c.x, c.residual, c.weight, c.post, c.sum, c.codes, c.scales}));
  // the sum may replace an addend in place: the same rows, element for element
  auto in_place = [&](const void *p, int64_t ld) { return c.sum && c.sum == p && (c.lds == ld || c.M == 1); };
  const Span x = in_place(c.x, c.ldx) ? Span{0, 0} : rows_of(c.x, c.M, c.ldx, c.K, 2);
  const Span r = in_place(c.residual, c.ldr) ? Span{0, 0} : rows_of(c.residual, c.M, c.ldr, c.K, 2);
  const Span sum = rows_of(c.sum, c.M, c.lds, c.K, 2), codes = span(c.codes, c.codes_bytes), scales = span(c.scales, c.scales_bytes);
  if (outputs_alias({sum, codes, scales}, {x, r, floats(c.weight, c.K), floats(c.post, c.K)}))
    return fail(FQ_ERR_ALIAS, "codes, scales and the sum must not overlap each other or an input (the sum may be an addend itself)");
  NormArgs a{};
  a.x = c.x;
  a.ldx = c.ldx;
  a.residual = c.residual;
  a.ldr = c.ldr;
  a.weight = c.weight;
  a.post = c.post;
  a.eps = c.eps;
  a.M = c.M;
  a.K = (int)c.K;
  a.b = c.b;
  a.clip_ratio = c.clip;
  a.cb = root_of(c.b);
  a.sum = c.sum;
  a.lds = c.lds;
  a.out_fmt = c.fmt;
  a.codes = static_cast<uint8_t *>(c.codes);
  if (c.fmt == kOutMx) a.scales = static_cast<uint8_t *>(c.scales);
  else a.delta = static_cast<float *>(c.scales);
  const hipError_t e = launch_norm_quant(a, static_cast<hipStream_t>(c.stream));
  return e == hipSuccess ? ok() : hip_fail(e, "norm launch");
}

fq_status check_quant(const char *ld, const float *pre, const float *post, int64_t ldx, int mult, int64_t M, int64_t K, int b) {
  FQ_TRY(check_rows("M", M));
  FQ_TRY(check_k(K));
  FQ_TRY(check_block(b, K));
  FQ_TRY(check_ld(ld, ldx, K, mult, M));
  return check_aligned({pre, post});
}

fq_status check_product(int64_t M, int64_t N, int64_t K, int64_t ldy) {
  FQ_TRY(check_rows("M", M));
  FQ_TRY(check_rows("N", N));
  FQ_TRY(check_k(K));
  if (N % 16) return fail(FQ_ERR_UNSUPPORTED, "N=%lld is not a multiple of 16", (long long)N);
  if (M * N > (1ll << 40)) return fail(FQ_ERR_UNSUPPORTED, "M x N = %lld outputs is too large", (long long)(M * N));
  return check_ld("ldy", ldy, N, 8, M);
}

MxQuantArgs quant_args(const void *x, bool f32, int64_t ldx, const float *pre, const float *post, int64_t M, int64_t K, int b,
                       void *codes, void *scales) {
  return MxQuantArgs{x, f32, ldx, pre, post, M, (int)K, b, root_of(b), static_cast<uint8_t *>(codes), static_cast<uint8_t *>(scales)};
}

fq_status pack_common(const void *from, int64_t N, int64_t K, bool unpack, void *to, void *stream) {
  FQ_TRY(check_rows("N", N));
  if (N % 16) return fail(FQ_ERR_UNSUPPORTED, "N=%lld is not a multiple of 16", (long long)N);
  FQ_TRY(check_k(K));
  if (N == 0) return ok();
  if (!from || !to) return fail(FQ_ERR_NULL, "codes and packed must be non-NULL");
  FQ_TRY(check_aligned({from, to}));
  if (overlap(span(from, mx_codes_bytes(N, K)), span(to, mx_codes_bytes(N, K))))
    return fail(FQ_ERR_ALIAS, "codes and packed must not overlap");
  const hipError_t e = launch_mx_pack(static_cast<const uint8_t *>(from), N, (int)K, unpack, static_cast<uint8_t *>(to),
                                      static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "mx pack launch");
}

fq_status read_common(const void *codes, const void *scale, int64_t M, int64_t K, int bits, void *values, int64_t ldv,
                      void *stream) {
  FQ_TRY(check_rows("M", M));
  FQ_TRY(check_k(K));
  FQ_TRY(check_ld("ldv", ldv, K, 8, M));
  if (M == 0) return ok();
  if (!codes || !scale || !values) return fail(FQ_ERR_NULL, "codes, scales and values must be non-NULL");
  FQ_TRY(check_aligned({codes, scale, values}));
  const size_t cb = bits == 8 ? (size_t)M * K : mx_codes_bytes(M, K), sb = bits ? (size_t)M * 4 : mx_scales_bytes(M, K);
  if (outputs_alias({rows_of(values, M, ldv, K, 2)}, {span(codes, cb), span(scale, sb)}))
    return fail(FQ_ERR_ALIAS, "values must not overlap the codes or the scales");
  const hipError_t e = launch_read_codes(static_cast<const uint8_t *>(codes), scale, M, (int)K, bits,
                                         static_cast<uint16_t *>(values), ldv, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "read launch");
}

bool product_sizes(int64_t M, int64_t N, int64_t K) {
  return M > 0 && N > 0 && M <= kMaxRows && N <= kMaxRows && K >= 128 && K <= kMaxK;
}

size_t linear_workspace(const MxPlan &p, int64_t M, int64_t N, int64_t K) {
  return p.token ? 0 : align256(mx_codes_bytes(M, K)) + align256(mx_scales_bytes(M, K)) + mx_gemm_workspace(p, M, N);
}

fq_status check_room(const void *ws, size_t have, size_t need) {
  if (need > 0 && (!ws || have < need))
    return fail(FQ_ERR_WORKSPACE, "workspace of %zu bytes needed, %zu given", need, ws ? have : (size_t)0);
  if (need > 0 && !aligned16(ws)) return fail(FQ_ERR_ALIGN, "workspace must be 16-byte aligned");
  return FQ_OK;
}

}  // namespace

extern "C" {

fq_status fq_norm_quant(const void *x_bf16, int64_t ldx, const void *residual_bf16, int64_t ldr, const float *weight, float eps,
                        const float *post_inv, int64_t M, int64_t K, int b, int bits, float clip_ratio, void *sum_out,
                        int64_t ld_sum, void *codes, float *delta, void *stream) {
  if (bits != 4 && bits != 8) return fail(FQ_ERR_UNSUPPORTED, "bits=%d (must be 4 or 8)", bits);
  return norm_common(NormCall{x_bf16, ldx, residual_bf16, ldr, weight, eps, post_inv, M, K, b, clip_ratio, sum_out, ld_sum, codes,
                              delta, M > 0 ? (size_t)M * (size_t)K * (size_t)bits / 8 : 0, M > 0 ? (size_t)M * 4 : 0,
                              bits == 4 ? kOutNibble : kOutInt8, stream});
}

fq_status fq_norm_mx_quant(const void *x_bf16, int64_t ldx, const void *residual_bf16, int64_t ldr, const float *weight, float eps,
                           const float *post_inv, int64_t M, int64_t K, int b, void *sum_out, int64_t ld_sum, void *codes,
                           void *scales, void *stream) {
  return norm_common(NormCall{x_bf16, ldx, residual_bf16, ldr, weight, eps, post_inv, M, K, b, 1.0f, sum_out, ld_sum, codes,
                              scales, M > 0 ? mx_codes_bytes(M, K) : 0, M > 0 ? mx_scales_bytes(M, K) : 0, kOutMx, stream});
}

fq_status fq_read_codes(const void *codes, const float *delta, int64_t M, int64_t K, int bits, void *values_bf16, int64_t ldv,
                        void *stream) {
  if (bits != 4 && bits != 8) return fail(FQ_ERR_UNSUPPORTED, "bits=%d (must be 4 or 8)", bits);
  return read_common(codes, delta, M, K, bits, values_bf16, ldv, stream);
}

fq_status fq_mx_quant(const void *x, int x_is_f32, int64_t ldx, const float *pre_mult, const float *post_mult, int64_t M,
                      int64_t K, int b, void *codes, void *scales, void *stream) {
  const int size = x_is_f32 ? 4 : 2;
  FQ_TRY(check_quant("ldx", pre_mult, post_mult, ldx, 16 / size, M, K, b));
  if (M == 0) return ok();
  if (!x || !codes || !scales) return fail(FQ_ERR_NULL, "x, codes and scales must be non-NULL");
  FQ_TRY(check_aligned({x, codes, scales}));
  if (outputs_alias({span(codes, mx_codes_bytes(M, K)), span(scales, mx_scales_bytes(M, K))},
                    {rows_of(x, M, ldx, K, size), floats(pre_mult, K), floats(post_mult, K)}))
    return fail(FQ_ERR_ALIAS, "codes and scales must not overlap each other or an input");
  const hipError_t e = launch_mx_quant(quant_args(x, x_is_f32 != 0, ldx, pre_mult, post_mult, M, K, b, codes, scales),
                                       static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "mx quantization launch");
}

fq_status fq_mx_read(const void *codes, const void *scales, int64_t M, int64_t K, void *values_bf16, int64_t ldv, void *stream) {
  return read_common(codes, scales, M, K, 0, values_bf16, ldv, stream);
}

size_t fq_mx_packed_bytes(int64_t N, int64_t K) { return N < 0 || K < 0 ? 0 : mx_codes_bytes(N, K); }

fq_status fq_mx_pack(const void *codes, int64_t N, int64_t K, void *packed, void *stream) {
  return pack_common(codes, N, K, false, packed, stream);
}

fq_status fq_mx_unpack(const void *packed, int64_t N, int64_t K, void *codes, void *stream) {
  return pack_common(packed, N, K, true, codes, stream);
}

size_t fq_mx_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  return !product_sizes(M, N, K) ? 0 : mx_gemm_workspace(mx_plan(M, N, K), M, N);
}

fq_status fq_mx_gemm(const void *a_codes, const void *a_scales, const void *w_packed, const void *w_scales, const float *bias,
                     void *y_bf16, int64_t ldy, int64_t M, int64_t N, int64_t K, void *ws, size_t ws_bytes, void *stream) {
  FQ_TRY(check_product(M, N, K, ldy));
  if (M == 0 || N == 0) return ok();
  if (!a_codes || !a_scales || !w_packed || !w_scales || !y_bf16)
    return fail(FQ_ERR_NULL, "a_codes, a_scales, w_packed, w_scales and y must be non-NULL");
  FQ_TRY(check_aligned({a_codes, a_scales, w_packed, w_scales, bias, y_bf16}));
  const MxPlan plan = mx_plan(M, N, K);
  const size_t need = mx_gemm_workspace(plan, M, N);
  FQ_TRY(check_room(ws, ws_bytes, need));
  if (outputs_alias({rows_of(y_bf16, M, ldy, N, 2), span(need ? ws : nullptr, need)},
                    {span(a_codes, mx_codes_bytes(M, K)), span(a_scales, mx_scales_bytes(M, K)), span(w_packed, mx_codes_bytes(N, K)),
                     span(w_scales, mx_scales_bytes(N, K)), floats(bias, N)}))
    return fail(FQ_ERR_ALIAS, "y and the workspace must not overlap each other or an input");
  const MxGemmArgs g{static_cast<const uint8_t *>(a_codes), static_cast<const uint8_t *>(a_scales),
                     static_cast<const uint8_t *>(w_packed), static_cast<const uint8_t *>(w_scales), bias,
                     static_cast<uint16_t *>(y_bf16), ldy, M, N, (int)K};
  const hipError_t e = launch_mx_gemm(g, plan, ws, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? ok() : hip_fail(e, "mx product launch");
}

size_t fq_mx_linear_workspace_bytes(int64_t M, int64_t N, int64_t K) {
  return !product_sizes(M, N, K) ? 0 : linear_workspace(mx_plan(M, N, K), M, N, K);
}

fq_status fq_mx_linear(const void *x_bf16, int64_t ldx, const float *smooth_inv, const float *post_inv, int64_t M, int64_t K,
                       int64_t N, int b, const void *w_packed, const void *w_scales, const float *bias, void *y_bf16, int64_t ldy,
                       void *ws, size_t ws_bytes, void *stream) {
  FQ_TRY(check_quant("ldx", smooth_inv, post_inv, ldx, 8, M, K, b));
  FQ_TRY(check_product(M, N, K, ldy));
  if (M == 0 || N == 0) return ok();
  if (!x_bf16 || !w_packed || !w_scales || !y_bf16) return fail(FQ_ERR_NULL, "x, w_packed, w_scales and y must be non-NULL");
  FQ_TRY(check_aligned({x_bf16, w_packed, w_scales, bias, y_bf16}));
  const MxPlan plan = mx_plan(M, N, K);
  const size_t need = linear_workspace(plan, M, N, K);
  FQ_TRY(check_room(ws, ws_bytes, need));
  if (outputs_alias({rows_of(y_bf16, M, ldy, N, 2), span(need ? ws : nullptr, need)},
                    {rows_of(x_bf16, M, ldx, K, 2), floats(smooth_inv, K), floats(post_inv, K), span(w_packed, mx_codes_bytes(N, K)),
                     span(w_scales, mx_scales_bytes(N, K)), floats(bias, N)}))
    return fail(FQ_ERR_ALIAS, "y and the workspace must not overlap each other or an input");
  // codes and scales of the workspace; a launch that rounds for itself has none
  uint8_t *codes = static_cast<uint8_t *>(ws), *scales = plan.token ? nullptr : codes + align256(mx_codes_bytes(M, K));
  const MxQuantArgs q = quant_args(x_bf16, false, ldx, smooth_inv, post_inv, M, K, b, codes, scales);
  const MxGemmArgs g{codes, scales, static_cast<const uint8_t *>(w_packed), static_cast<const uint8_t *>(w_scales), bias,
                     static_cast<uint16_t *>(y_bf16), ldy, M, N, (int)K};
  hipStream_t st = static_cast<hipStream_t>(stream);
  hipError_t e;
  if (plan.token) {
    e = launch_mx_token(q, g, plan, st);
  } else {
    e = launch_mx_quant(q, st);
    if (e == hipSuccess) e = launch_mx_gemm(g, plan, scales + align256(mx_scales_bytes(M, K)), st);
  }
  return e == hipSuccess ? ok() : hip_fail(e, "mx projection launch");
}

}  // extern "C"
