// C ABI of the operators around a protected classifier (include/ctc.h):
// checks the arguments, then enqueues the kernels of ops.hip.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/ctc.h"
#include "errors.h"
#include "ops.h"

using namespace ctc::ops;

namespace {

ctc_status fail(ctc_status s, const char *fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return ctc::report(s, buf);
}
ctc_status done(hipError_t e) {
    return e == hipSuccess ? CTC_OK : fail(CTC_ERR_DEVICE, "%s", hipGetErrorString(e));
}
hipStream_t S(void *s) { return (hipStream_t)s; }

bool real_type(int t) { return t == CTC_F32 || t == CTC_F16 || t == CTC_BF16; }
bool byte_type(int t) { return t == CTC_E4M3 || t == CTC_E5M2; }
bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
// A launch along one dimension takes fewer than 2^32 threads, and the largest
// workgroups of the quantiser, the product and the scores have 512.  (Those of
// the group norm have 1024, in grids of two dimensions.)
bool grid_ok(double workgroups) { return workgroups < 8388608.0; }

ctc_status need_workspace(size_t need, const void *ws, size_t bytes) {
    if (!need) return CTC_OK;
    if (!ws || bytes < need)
        return fail(CTC_ERR_WORKSPACE, "workspace of %zu bytes needed, got %zu", need,
                    ws ? bytes : (size_t)0);
    if (!aligned(ws, 16)) return fail(CTC_ERR_ARG, "workspace must be 16-byte aligned");
    return CTC_OK;
}

// ------------------------------------------------------------- group norm

ctc_status norm_args(ctc_dtype dtype, int32_t n, int64_t hw, int32_t c, int32_t groups,
                     int32_t carry, int32_t act, NormArgs &a) {
    if (!real_type(dtype)) return fail(CTC_ERR_ARG, "bad dtype");
    if (n < 0 || hw < 1 || c < 1) return fail(CTC_ERR_ARG, "bad group_norm sizes");
    if (groups < 1 || c % groups) return fail(CTC_ERR_ARG, "groups must divide c");
    if (act < CTC_ACT_NONE || act > CTC_ACT_SILU) return fail(CTC_ERR_ARG, "bad activation");
    if (hw > ((int64_t)1 << 31) || c > (1 << 20))
        return fail(CTC_ERR_UNSUPPORTED, "maps of up to 2^31 pixels and 2^20 channels");
    // (workgroups have numbers of 32 bits; there are at most n * c of them, or
    // 2048)
    if ((int64_t)n * c >> 32) return fail(CTC_ERR_UNSUPPORTED, "too many images");
    a = NormArgs{};
    a.type = dtype; a.n = n; a.hw = hw; a.c = c; a.groups = groups;
    a.carry = carry != 0; a.act = act;
    return CTC_OK;
}

// -------------------------------------------------------------- quantiser

ctc_status matrix_8bit(const void *q, int64_t rows, int64_t cols, int64_t ld) {
    if (rows && cols && !q) return fail(CTC_ERR_ARG, "NULL matrix");
    if (ld < (cols + 15) / 16 * 16 || ld % 16 || !aligned(q, 16))
        return fail(CTC_ERR_ARG, "8-bit rows must begin at multiples of 16 bytes and "
                    "hold their columns rounded up to 16");
    return CTC_OK;
}

ctc_status product_args(ctc_dtype atype, ctc_dtype btype, ctc_dtype ytype, int64_t m, int64_t n,
                        int64_t k, int32_t a_block, int32_t b_block, ProductArgs &p) {
    if (!byte_type(atype) || !byte_type(btype) || !real_type(ytype))
        return fail(CTC_ERR_ARG, "bad dtype");
    if (m < 0 || n < 0 || k < 0) return fail(CTC_ERR_ARG, "bad product sizes");
    if ((a_block != 1 && a_block != 128) || (b_block != 1 && b_block != 128))
        return fail(CTC_ERR_ARG, "a scale holds for 1 or 128 rows");
    if (m > (1 << 30) || n > (1 << 30) || k > (1 << 30) ||
        !grid_ok((double)m * ((double)n / 4 + 1) / 256 + 1) ||
        !grid_ok((double)n / 16 * 16 + 1))
        return fail(CTC_ERR_UNSUPPORTED, "product too large");
    p = ProductArgs{};
    p.atype = atype; p.btype = btype; p.ytype = ytype;
    p.m = m; p.n = n; p.k = k; p.a_block = a_block; p.b_block = b_block;
    return CTC_OK;
}

// ----------------------------------------------------------------- scores

ctc_status score_args(ctc_dtype dtype, int64_t rows, int32_t vocab, int64_t ld, int32_t top_k,
                      ScoreArgs &a) {
    if (!real_type(dtype)) return fail(CTC_ERR_ARG, "bad dtype");
    if (rows < 0 || vocab < 1 || ld < vocab) return fail(CTC_ERR_ARG, "bad token_scores sizes");
    if (top_k < 0 || top_k > SCORES_MAX_K)
        return fail(CTC_ERR_ARG, "top_k must be 0 .. %d", SCORES_MAX_K);
    if (vocab > (1 << 30) || !grid_ok((double)rows) ||
        !grid_ok((double)rows * ((double)vocab / 4096 + 1)))
        return fail(CTC_ERR_UNSUPPORTED, "too many rows");
    a = ScoreArgs{};
    a.type = dtype; a.rows = rows; a.ld = ld; a.vocab = vocab; a.top_k = top_k;
    return CTC_OK;
}

}  // namespace

extern "C" {

ctc_status ctc_group_norm_workspace_bytes(ctc_dtype dtype, int32_t n, int64_t hw, int32_t c,
                                          int32_t groups, int32_t backward, size_t *bytes) {
    if (!bytes) return fail(CTC_ERR_ARG, "NULL bytes");
    NormArgs a;
    ctc_status s = norm_args(dtype, n, hw, c, groups, 0, 0, a);
    if (s != CTC_OK) return s;
    *bytes = norm_workspace(a, backward != 0);
    return CTC_OK;
}

ctc_status ctc_group_norm_forward(ctc_dtype dtype, int32_t n, int64_t hw, int32_t c,
                                  int32_t groups, int32_t carry, const void *x,
                                  const float *gamma, const float *beta, const void *residual,
                                  float eps, int32_t act, void *y, float *mean, float *rstd,
                                  void *workspace, size_t ws_bytes, void *stream) {
    NormArgs a;
    ctc_status s = norm_args(dtype, n, hw, c, groups, carry, act, a);
    if (s != CTC_OK) return s;
    if (!(eps >= 0.f) || std::isinf(eps)) return fail(CTC_ERR_ARG, "bad eps");
    if (n == 0) return CTC_OK;
    if (!x || !y || !mean || !rstd) return fail(CTC_ERR_ARG, "bad group_norm arguments");
    a.x = x; a.gamma = gamma; a.beta = beta; a.residual = residual; a.eps = eps;
    a.y = y; a.mean = mean; a.rstd = rstd; a.ws = (float *)workspace;
    s = need_workspace(norm_workspace(a, false), workspace, ws_bytes);
    if (s != CTC_OK) return s;
    return done(launch_norm_forward(a, S(stream)));
}

ctc_status ctc_group_norm_backward(ctc_dtype dtype, int32_t n, int64_t hw, int32_t c,
                                   int32_t groups, int32_t carry, const void *dy, const void *x,
                                   const float *mean, const float *rstd, const float *gamma,
                                   const float *beta, const void *residual, int32_t act,
                                   void *dx, void *dresidual, float *dgamma, float *dbeta,
                                   void *workspace, size_t ws_bytes, void *stream) {
    NormArgs a;
    ctc_status s = norm_args(dtype, n, hw, c, groups, carry, act, a);
    if (s != CTC_OK) return s;
    if (n && (!dy || !x || !mean || !rstd))
        return fail(CTC_ERR_ARG, "bad group_norm_backward arguments");
    a.x = x; a.gamma = gamma; a.beta = beta; a.residual = residual; a.dy = dy;
    a.dx = dx; a.dresidual = dresidual; a.dgamma = dgamma; a.dbeta = dbeta;
    a.mean = (float *)mean; a.rstd = (float *)rstd; a.ws = (float *)workspace;
    s = need_workspace(n ? norm_workspace(a, true) : 0, workspace, ws_bytes);
    if (s != CTC_OK) return s;
    return done(launch_norm_backward(a, S(stream)));
}

ctc_status ctc_fp8_quantize(ctc_dtype dtype, int64_t rows, int64_t cols, const void *x,
                            int64_t ldx, ctc_dtype qtype, int32_t block_rows, int32_t transpose,
                            void *q, int64_t ldq, float *scales, int64_t ld_scales,
                            void *stream) {
    if (!real_type(dtype) || !byte_type(qtype)) return fail(CTC_ERR_ARG, "bad dtype");
    if (rows < 0 || cols < 0 || ldx < cols) return fail(CTC_ERR_ARG, "bad fp8_quantize sizes");
    if (block_rows != 1 && block_rows != 128)
        return fail(CTC_ERR_ARG, "a scale holds for 1 or 128 rows");
    if (!grid_ok(((double)rows / 16 + 1) * ((double)cols / 128 + 1)))
        return fail(CTC_ERR_UNSUPPORTED, "matrix too large");
    if (rows == 0 || cols == 0) return CTC_OK;
    if (!x || !scales) return fail(CTC_ERR_ARG, "bad fp8_quantize arguments");
    const int64_t qr = transpose ? cols : rows, qc = transpose ? rows : cols;
    ctc_status s = matrix_8bit(q, qr, qc, ldq);
    if (s != CTC_OK) return s;
    if (ld_scales < (qr + block_rows - 1) / block_rows)
        return fail(CTC_ERR_ARG, "ld_scales below the number of row blocks");
    QuantArgs a{};
    a.type = dtype; a.qtype = qtype; a.rows = rows; a.cols = cols; a.ldx = ldx;
    a.transpose = transpose != 0; a.block_rows = block_rows;
    a.x = x; a.q = (uint8_t *)q; a.ldq = ldq; a.scales = scales; a.lds = ld_scales;
    return done(launch_quantize(a, S(stream)));
}

ctc_status ctc_fp8_matmul_workspace_bytes(ctc_dtype ytype, int64_t m, int64_t n, int64_t k,
                                          int32_t b_block, size_t *bytes) {
    if (!bytes) return fail(CTC_ERR_ARG, "NULL bytes");
    ProductArgs p;
    ctc_status s = product_args(CTC_E4M3, CTC_E4M3, ytype, m, n, k, 1, b_block, p);
    if (s != CTC_OK) return s;
    *bytes = m && n ? product_workspace(p) : 0;
    return CTC_OK;
}

ctc_status ctc_fp8_matmul(ctc_dtype atype, ctc_dtype btype, ctc_dtype ytype, int64_t m,
                          int64_t n, int64_t k, const void *a, int64_t lda,
                          const float *a_scales, int64_t ld_as, int32_t a_block, const void *b,
                          int64_t ldb, const float *b_scales, int64_t ld_bs, int32_t b_block,
                          const float *bias, int32_t act, void *y, int64_t ldy, void *workspace,
                          size_t ws_bytes, void *stream) {
    ProductArgs p;
    ctc_status s = product_args(atype, btype, ytype, m, n, k, a_block, b_block, p);
    if (s != CTC_OK) return s;
    if (act < CTC_ACT_NONE || act > CTC_ACT_SILU) return fail(CTC_ERR_ARG, "bad activation");
    if (ldy < n) return fail(CTC_ERR_ARG, "ldy below n");
    if (lda > (1 << 22) || ldb > (1 << 22))
        return fail(CTC_ERR_UNSUPPORTED, "rows of up to 2^22 bytes");
    if (m == 0 || n == 0) return CTC_OK;
    if (!y || (k && (!a_scales || !b_scales)))
        return fail(CTC_ERR_ARG, "bad fp8_matmul arguments");
    s = matrix_8bit(a, m, k, lda);
    if (s == CTC_OK) s = matrix_8bit(b, n, k, ldb);
    if (s != CTC_OK) return s;
    if (k && (ld_as < (m + a_block - 1) / a_block || ld_bs < (n + b_block - 1) / b_block))
        return fail(CTC_ERR_ARG, "scales' stride below the number of row blocks");
    p.act = act; p.a = (const uint8_t *)a; p.b = (const uint8_t *)b;
    p.lda = lda; p.ldb = ldb; p.ldy = ldy; p.sa = a_scales; p.sb = b_scales;
    p.ldsa = ld_as; p.ldsb = ld_bs; p.bias = bias; p.y = y; p.ws = (float *)workspace;
    s = need_workspace(product_workspace(p), workspace, ws_bytes);
    if (s != CTC_OK) return s;
    return done(launch_product(p, S(stream)));
}

ctc_status ctc_token_scores_workspace_bytes(int64_t rows, int32_t vocab, int32_t top_k,
                                            size_t *bytes) {
    if (!bytes) return fail(CTC_ERR_ARG, "NULL bytes");
    ScoreArgs a;
    ctc_status s = score_args(CTC_F32, rows, vocab, vocab, top_k, a);
    if (s != CTC_OK) return s;
    *bytes = scores_workspace(a);
    return CTC_OK;
}

ctc_status ctc_token_scores_forward(ctc_dtype dtype, int64_t rows, int32_t vocab,
                                    const void *logits, int64_t ld, const int32_t *targets,
                                    int32_t top_k, float *lse, float *logprob, float *entropy,
                                    int32_t *rank, int32_t *top_ids, float *top_logprobs,
                                    void *workspace, size_t ws_bytes, void *stream) {
    ScoreArgs a;
    ctc_status s = score_args(dtype, rows, vocab, ld, top_k, a);
    if (s != CTC_OK) return s;
    if (rows == 0) return CTC_OK;
    if (!logits) return fail(CTC_ERR_ARG, "NULL logits");
    if ((logprob || rank) && !targets) return fail(CTC_ERR_ARG, "logprob and rank need targets");
    if (top_k && (!top_ids || !top_logprobs))
        return fail(CTC_ERR_ARG, "top_k without top_ids and top_logprobs");
    a.x = logits; a.target = targets; a.lse = lse; a.logprob = logprob;
    a.entropy = entropy; a.rank = rank; a.ids = top_ids; a.tops = top_logprobs;
    a.ws = workspace;
    s = need_workspace(scores_workspace(a), workspace, ws_bytes);
    if (s != CTC_OK) return s;
    return done(launch_scores(a, S(stream)));
}

ctc_status ctc_token_scores_backward(ctc_dtype dtype, int64_t rows, int32_t vocab,
                                     const void *logits, int64_t ld, const int32_t *targets,
                                     const float *lse, const float *entropy, const float *g_lse,
                                     const float *g_logprob, const float *g_entropy,
                                     void *dlogits, int64_t ldd, void *stream) {
    ScoreArgs a;
    ctc_status s = score_args(dtype, rows, vocab, ld, 0, a);
    if (s != CTC_OK) return s;
    if (ldd < vocab) return fail(CTC_ERR_ARG, "ldd below vocab");
    if (rows == 0) return CTC_OK;
    if (!logits || !lse || !dlogits) return fail(CTC_ERR_ARG, "bad token_scores_backward arguments");
    if (g_logprob && !targets) return fail(CTC_ERR_ARG, "g_logprob needs targets");
    if (g_entropy && !entropy) return fail(CTC_ERR_ARG, "g_entropy needs the entropy");
    if (dlogits == logits && ldd != ld)
        return fail(CTC_ERR_ARG, "dlogits in place needs the logits' stride");
    a.x = logits; a.target = targets; a.lse = (float *)lse; a.entropy = (float *)entropy;
    a.g_lse = g_lse; a.g_logprob = g_logprob; a.g_entropy = g_entropy;
    a.dx = dlogits; a.ldd = ldd;
    return done(launch_scores_backward(a, S(stream)));
}

}  // extern "C"
