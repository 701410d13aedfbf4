// The experts of many tokens: rows in expert order through a gated two-layer network in
// 8-bit products.
//
//   quantise (through the gather map) -> gate and up product, SwiGLU, 8-bit result ->
//   down product -> weighted sum back into token order
//
// The widest intermediate, two products of `inter` columns a row, is never written: the
// first product's epilogue turns it into 8-bit rows (tuna_fp8.cu).
//
// An expert's row is rounded to bf16 (2^-9 of each value) before the weighted sum, which adds in 32 bits.  It is the
// row that tuna_moe_expert_rows hands to the return of a token dispatch, so that a layer gives the same bits with its
// experts in place and behind an exchange; and in 32 bits it would be written and read at twice the bytes
// (268 MB more for 8192 tokens x 2 slots of 4096 columns, 41 us at 6552 GB/s).  For a few tokens the traffic would be
// nothing, and the one reason is that the bits are the same.  What it costs: two slots in bf16 and the sum's own
// rounding are off by 0.0023 to 0.0024 of the result (root of the mean square against 64 bits), one rounding alone by 0.0017.
//
// With 4-bit weights (tuna_fp4.cu) the steps are the same, x and h in 4 bits too, and so are the rounding and its reasons.
#include "tuna_fp4.h"
#include "tuna_fp8.h"
#include "tuna_ops.cuh"

namespace tuna_ops {
namespace {

struct RowsSpace {
  uint8_t *q, *h;
  float *qs, *hs;
  int64_t ldq, ldh;
};
RowsSpace carve_rows(Carve &c, int64_t rows, int hidden, int inter) {
  RowsSpace w = {};
  w.ldq = ceil_div(hidden, 16) * 16;
  w.ldh = ceil_div(inter, 128) * 128;  // whole blocks: the first product stores them unmasked
  w.q = c.take<uint8_t>(rows * w.ldq);
  w.h = c.take<uint8_t>(rows * w.ldh);
  w.qs = c.take<float>(rows * ceil_div(hidden, 128));
  w.hs = c.take<float>(rows * ceil_div(inter, 128));
  return w;
}

int check_experts(int64_t rows, int experts, int hidden, int inter) {
  if (rows < 0 || experts < 1 || hidden < 1 || inter < 1 || hidden % 16 || inter % 16) return TUNA_ERR_INVALID_ARG;
  if (experts > TUNA_MOE_MAX_EXPERTS || hidden > (1 << 20) || inter > (1 << 20) || rows > (1 << 24)) return TUNA_ERR_RANGE;
  return TUNA_OK;
}

int run_rows(const void *x, int64_t ldx, int64_t rows, const int64_t *gather, int64_t in_rows, int experts, const int64_t *offsets, int hidden,
             int inter, const void *w13, const float *s13, const void *w2, const float *s2, void *y, int64_t ldy, const RowsSpace &w,
             cudaStream_t st) {
  if (const int rc = launch_quantize_rows(x, false, rows, hidden, ldx, gather, in_rows, w.q, w.ldq, w.qs, st)) return rc;
  ProductArgs p = {};
  p.a = w.q, p.sa = w.qs, p.b = w13, p.sb = s13, p.m = rows, p.n = inter, p.k = hidden, p.lda = w.ldq, p.ldb = hidden;
  p.groups = experts, p.offsets = offsets, p.out = w.h, p.ldo = w.ldh, p.hs = w.hs, p.swiglu = true;
  if (const int rc = launch_product(p, st)) return rc;
  p = {};
  p.a = w.h, p.sa = w.hs, p.b = w2, p.sb = s2, p.m = rows, p.n = hidden, p.k = inter, p.lda = w.ldh, p.ldb = inter;
  p.groups = experts, p.offsets = offsets, p.out = y, p.ldo = ldy;
  return launch_product(p, st);
}

struct TokenSpace {
  RowsSpace rows;
  int64_t *offsets, *order, *pos;
  uint16_t *y;
  char *sort;
  size_t sort_bytes;
};
TokenSpace carve_tokens(Carve &c, int64_t tokens, int experts, int k, int hidden, int inter) {
  TokenSpace w = {};
  const int64_t n = tokens * k;
  w.rows = carve_rows(c, n, hidden, inter);
  w.offsets = c.take<int64_t>(experts + 1);
  w.order = c.take<int64_t>(n);
  w.pos = c.take<int64_t>(n);
  w.y = c.take<uint16_t>(n * hidden);
  w.sort_bytes = 0;
  tuna_moe_order_workspace_bytes(tokens, experts, k, 1, &w.sort_bytes);
  w.sort = c.take<char>((int64_t)w.sort_bytes);
  return w;
}

// ---- 4-bit weights ----

struct Rows4Space {
  uint8_t *q, *h, *qs, *hs;
  int64_t ldq, ldh;
};
Rows4Space carve_rows4(Carve &c, int64_t rows, int experts, int hidden, int inter) {
  Rows4Space w = {};
  const int64_t tiles = fp4_slots(rows, experts);
  w.ldq = hidden / 2;
  w.ldh = ceil_div(inter, 128) * 64;  // whole tiles: the first product stores them unmasked
  w.q = c.take<uint8_t>(rows * w.ldq);
  w.h = c.take<uint8_t>(rows * w.ldh);
  w.qs = c.take<uint8_t>(tiles * ceil_div(hidden, 128) * kScaleTile);
  w.hs = c.take<uint8_t>(tiles * ceil_div(inter, 128) * kScaleTile);
  return w;
}

int check_experts4(int64_t rows, int experts, int hidden, int inter) {
  if (hidden % 32 || inter % 32) return TUNA_ERR_INVALID_ARG;
  return check_experts(rows, experts, hidden, inter);
}

// The two products of quantised rows.
int run_products4(int64_t rows, int experts, const int64_t *offsets, int hidden, int inter, const void *w13, const void *s13, const void *w2,
                  const void *s2, void *y, int64_t ldy, const Rows4Space &w, cudaStream_t st) {
  Product4Args p = {};
  p.a = w.q, p.sa = w.qs, p.b = w13, p.sb = (const uint8_t *)s13, p.m = rows, p.n = inter, p.k = hidden, p.lda = w.ldq, p.ldb = hidden / 2;
  p.groups = experts, p.offsets = offsets, p.out = w.h, p.ldo = w.ldh, p.hs = w.hs, p.swiglu = true;
  if (const int rc = launch_product4(p, st)) return rc;
  p = {};
  p.a = w.h, p.sa = w.hs, p.b = w2, p.sb = (const uint8_t *)s2, p.m = rows, p.n = hidden, p.k = inter, p.lda = w.ldh, p.ldb = inter / 2;
  p.groups = experts, p.offsets = offsets, p.out = y, p.ldo = ldy;
  return launch_product4(p, st);
}

struct Token4Space {
  Rows4Space rows;
  int64_t *offsets, *order, *pos;
  uint16_t *y;
  char *sort;
  size_t sort_bytes;
};
Token4Space carve_tokens4(Carve &c, int64_t tokens, int experts, int k, int hidden, int inter) {
  Token4Space w = {};
  const int64_t n = tokens * k;
  w.rows = carve_rows4(c, n, experts, hidden, inter);
  w.offsets = c.take<int64_t>(experts + 1);
  w.order = c.take<int64_t>(n);
  w.pos = c.take<int64_t>(n);
  w.y = c.take<uint16_t>(n * hidden);
  tuna_moe_order_workspace_bytes(tokens, experts, k, 1, &w.sort_bytes);
  w.sort = c.take<char>((int64_t)w.sort_bytes);
  return w;
}

}  // namespace
}  // namespace tuna_ops

using namespace tuna_ops;

extern "C" {

int tuna_moe_expert_rows_workspace_bytes(int64_t rows, int hidden, int inter, size_t *bytes) {
  if (!bytes) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_experts(rows, 1, hidden, inter)) return rc;
  Carve c(nullptr);
  carve_rows(c, rows, hidden, inter);
  *bytes = c.used;
  return TUNA_OK;
}

int tuna_moe_expert_rows(const void *x, int64_t ldx, int64_t rows, int experts, const int64_t *offsets, int hidden, int inter, const void *w13,
                         const float *s13, const void *w2, const float *s2, void *y, int64_t ldy, void *workspace, size_t workspace_bytes,
                         void *stream) {
  if (const int rc = check_experts(rows, experts, hidden, inter)) return rc;
  if (ldx < hidden || ldy < hidden) return TUNA_ERR_INVALID_ARG;
  if (rows == 0) return TUNA_OK;
  if (!x || !offsets || !w13 || !s13 || !w2 || !s2 || !y || !aligned(x, 2) || !aligned(y, 2) || !aligned(w13, 16) || !aligned(w2, 16)) return TUNA_ERR_INVALID_ARG;
  Carve c(workspace);
  const RowsSpace w = carve_rows(c, rows, hidden, inter);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < c.used) return TUNA_ERR_WORKSPACE;
  return run_rows(x, ldx, rows, nullptr, rows, experts, offsets, hidden, inter, w13, s13, w2, s2, y, ldy, w, (cudaStream_t)stream);
}

int tuna_moe_experts_workspace_bytes(int64_t tokens, int experts, int k, int hidden, int inter, size_t *bytes) {
  if (!bytes || k < 1 || k > experts) return TUNA_ERR_INVALID_ARG;
  if (tokens < 0 || tokens > (1 << 24) || k > TUNA_MOE_MAX_K) return tokens < 0 ? TUNA_ERR_INVALID_ARG : TUNA_ERR_RANGE;
  if (const int rc = check_experts(tokens * k, experts, hidden, inter)) return rc;
  Carve c(nullptr);
  carve_tokens(c, tokens, experts, k, hidden, inter);
  *bytes = c.used;
  return TUNA_OK;
}

int tuna_moe_experts(const void *x, int64_t ldx, int64_t tokens, const int32_t *ids, const float *weights, int k, int experts, int hidden,
                     int inter, const void *w13, const float *s13, const void *w2, const float *s2, void *out, int64_t ldo, void *workspace,
                     size_t workspace_bytes, void *stream) {
  size_t need = 0;
  if (const int rc = tuna_moe_experts_workspace_bytes(tokens, experts, k, hidden, inter, &need)) return rc;
  if (ldx < hidden || ldo < hidden) return TUNA_ERR_INVALID_ARG;
  if (tokens == 0) return TUNA_OK;
  if (!x || !ids || !weights || !w13 || !s13 || !w2 || !s2 || !out || !aligned(x, 2) || !aligned(out, 2) || !aligned(w13, 16) || !aligned(w2, 16))
    return TUNA_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return TUNA_ERR_WORKSPACE;
  Carve c(workspace);
  const TokenSpace w = carve_tokens(c, tokens, experts, k, hidden, inter);
  if (const int rc = tuna_moe_order(ids, tokens, experts, k, 1, nullptr, w.offsets, w.order, w.pos, w.sort, w.sort_bytes, stream)) return rc;
  if (const int rc = run_rows(x, ldx, tokens * k, w.order, tokens, experts, w.offsets, hidden, inter, w13, s13, w2, s2, w.y, hidden, w.rows,
                              (cudaStream_t)stream))
    return rc;
  return tuna_moe_combine(w.y, TUNA_DTYPE_BF16, tokens * k, hidden, hidden, weights, w.pos, tokens, k, out, TUNA_DTYPE_BF16, ldo, stream);
}

int tuna_fp4_expert_rows_workspace_bytes(int64_t rows, int experts, int hidden, int inter, size_t *bytes) {
  if (!bytes) return TUNA_ERR_INVALID_ARG;
  if (const int rc = check_experts4(rows, experts, hidden, inter)) return rc;
  Carve c(nullptr);
  carve_rows4(c, rows, experts, hidden, inter);
  *bytes = c.used;
  return TUNA_OK;
}

int tuna_fp4_expert_rows(const void *x, int64_t ldx, int64_t rows, int experts, const int64_t *offsets, int hidden, int inter, const void *w13,
                         const void *s13, const void *w2, const void *s2, void *y, int64_t ldy, void *workspace, size_t workspace_bytes,
                         void *stream) {
  if (const int rc = check_experts4(rows, experts, hidden, inter)) return rc;
  if (ldx < hidden || ldy < hidden) return TUNA_ERR_INVALID_ARG;
  if (rows == 0) return TUNA_OK;
  if (!x || !offsets || !w13 || !s13 || !w2 || !s2 || !y || !aligned(x, 2) || !aligned(y, 2) || !aligned(offsets, 8) || !aligned(w13, 16) ||
      !aligned(s13, 16) || !aligned(w2, 16) || !aligned(s2, 16))
    return TUNA_ERR_INVALID_ARG;
  Carve c(workspace);
  const Rows4Space w = carve_rows4(c, rows, experts, hidden, inter);
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < c.used) return TUNA_ERR_WORKSPACE;
  cudaStream_t st = (cudaStream_t)stream;
  if (const int rc = launch_quantize4_rows(x, false, rows, hidden, ldx, nullptr, rows, experts, offsets, w.q, w.ldq, w.qs, st)) return rc;
  return run_products4(rows, experts, offsets, hidden, inter, w13, s13, w2, s2, y, ldy, w, st);
}

int tuna_fp4_experts_workspace_bytes(int64_t tokens, int experts, int k, int hidden, int inter, size_t *bytes) {
  if (!bytes || k < 1 || k > experts) return TUNA_ERR_INVALID_ARG;
  if (tokens < 0 || tokens > (1 << 24) || k > TUNA_MOE_MAX_K) return tokens < 0 ? TUNA_ERR_INVALID_ARG : TUNA_ERR_RANGE;
  if (const int rc = check_experts4(tokens * k, experts, hidden, inter)) return rc;
  Carve c(nullptr);
  carve_tokens4(c, tokens, experts, k, hidden, inter);
  *bytes = c.used;
  return TUNA_OK;
}

int tuna_fp4_experts(const void *x, int64_t ldx, int64_t tokens, const int32_t *ids, const float *weights, int k, int experts, int hidden,
                     int inter, const void *w13, const void *s13, const void *w2, const void *s2, void *out, int64_t ldo, void *workspace,
                     size_t workspace_bytes, void *stream) {
  size_t need = 0;
  if (const int rc = tuna_fp4_experts_workspace_bytes(tokens, experts, k, hidden, inter, &need)) return rc;
  if (ldx < hidden || ldo < hidden) return TUNA_ERR_INVALID_ARG;
  if (tokens == 0) return TUNA_OK;
  if (!x || !ids || !weights || !w13 || !s13 || !w2 || !s2 || !out || !aligned(x, 2) || !aligned(out, 2) || !aligned(ids, 4) || !aligned(weights, 4) ||
      !aligned(w13, 16) || !aligned(s13, 16) || !aligned(w2, 16) || !aligned(s2, 16))
    return TUNA_ERR_INVALID_ARG;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < need) return TUNA_ERR_WORKSPACE;
  Carve c(workspace);
  const Token4Space w = carve_tokens4(c, tokens, experts, k, hidden, inter);
  cudaStream_t st = (cudaStream_t)stream;
  if (places_quantize4(tokens * k)) {
    if (const int rc = launch_place_quantize4(x, tokens, hidden, ldx, ids, k, experts, w.rows.q, w.rows.ldq, w.rows.qs, w.offsets, w.pos, st)) return rc;
  } else {
    if (const int rc = tuna_moe_order(ids, tokens, experts, k, 1, nullptr, w.offsets, w.order, w.pos, w.sort, w.sort_bytes, stream)) return rc;
    if (const int rc = launch_quantize4_rows(x, false, tokens * k, hidden, ldx, w.order, tokens, experts, w.offsets, w.rows.q, w.rows.ldq, w.rows.qs, st))
      return rc;
  }
  if (const int rc = run_products4(tokens * k, experts, w.offsets, hidden, inter, w13, s13, w2, s2, w.y, hidden, w.rows, st)) return rc;
  return tuna_moe_combine(w.y, TUNA_DTYPE_BF16, tokens * k, hidden, hidden, weights, w.pos, tokens, k, out, TUNA_DTYPE_BF16, ldo, stream);
}

}  // extern "C"
