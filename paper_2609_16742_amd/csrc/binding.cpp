// Python binding of the operators around a protected classifier: checks
// torch tensors, allocates outputs and workspaces, calls the C ABI
// (include/ctc.h).  Marshalling only, compiled because an operator on a
// small batch runs for five microseconds and the same checks in Python took
// ten.  No torch types cross the C ABI: this is its caller.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/utils/pybind.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>

#include <array>
#include <cmath>
#include <optional>
#include <stdexcept>
#include <string>
#include <tuple>
#include <vector>

#include "../../include/ctc.h"

namespace py = pybind11;
using at::Tensor;
typedef std::optional<Tensor> Maybe;

namespace {

py::object check_status;         // ctc._check: raises CtcError

void done(ctc_status s) {
    if (s != CTC_OK) check_status((int)s);
}
void need(bool ok, const char *msg) {
    if (!ok) throw std::invalid_argument(msg);       // ValueError
}
void need(bool ok, const std::string &msg) {
    if (!ok) throw std::invalid_argument(msg);
}

bool real_type(const Tensor &t) {
    return t.scalar_type() == at::kFloat || t.scalar_type() == at::kHalf ||
           t.scalar_type() == at::kBFloat16;
}
bool byte_type(const Tensor &t) {
    return t.scalar_type() == at::kFloat8_e4m3fn || t.scalar_type() == at::kFloat8_e5m2;
}
ctc_dtype code(const Tensor &t) {
    switch (t.scalar_type()) {
    case at::kFloat: return CTC_F32;
    case at::kHalf: return CTC_F16;
    case at::kBFloat16: return CTC_BF16;
    case at::kFloat8_e4m3fn: return CTC_E4M3;
    default: return CTC_E5M2;
    }
}
void on_gpu(const Tensor &t, const char *name) {
    if (!t.defined() || !t.is_cuda())
        throw std::invalid_argument(std::string(name) + " must be a GPU tensor");
}
// Address of a contiguous tensor of that type, shape and device (or null).
template <size_t N>
void *like(const Maybe &t, const char *name, at::ScalarType type,
           const std::array<int64_t, N> &shape, const Tensor &ref) {
    if (!t) return nullptr;
    if (t->scalar_type() != type || t->sizes() != at::IntArrayRef(shape) ||
        t->device() != ref.device() || !t->is_contiguous())
        throw std::invalid_argument(
            std::string(name) + " must be a contiguous tensor of type " +
            c10::toString(type) + " and shape " + c10::str(at::IntArrayRef(shape)) + " on " +
            ref.device().str());
    return t->data_ptr();
}
void *like(const Maybe &t, const char *name, const Tensor &ref) {
    if (!t) return nullptr;
    if (t->scalar_type() != ref.scalar_type() || t->sizes() != ref.sizes() ||
        t->device() != ref.device() || !t->is_contiguous())
        throw std::invalid_argument(std::string(name) + " must be contiguous and like x");
    return t->data_ptr();
}
// Row stride of a matrix whose rows are contiguous.
int64_t rows_of(const Tensor &t, const char *name, const Tensor &ref) {
    if (t.dim() != 2 || t.device() != ref.device())
        throw std::invalid_argument(std::string(name) + " must be a matrix on " +
                                    ref.device().str());
    if (t.size(1) > 1 && t.stride(1) != 1)
        throw std::invalid_argument(std::string("the rows of ") + name + " must be contiguous");
    // (torch keeps no meaningful stride for a single row)
    if (t.size(0) <= 1) return t.size(1);
    if (t.stride(0) < t.size(1))
        throw std::invalid_argument(std::string("the rows of ") + name + " overlap");
    return t.stride(0);
}
// ... of an 8-bit matrix, all of whose rows can be read (and written) up to
// the next multiple of 16 columns.
int64_t rows_8bit(const Tensor &t, const char *name, const Tensor &ref) {
    int64_t ld = rows_of(t, name, ref);
    const int64_t wide = (t.size(1) + 15) / 16 * 16;
    if (t.size(0) == 0 || t.size(1) == 0) return wide;
    if (t.size(0) == 1) ld = wide;
    if (ld % 16 || (uintptr_t)t.data_ptr() % 16)
        throw std::invalid_argument(std::string("the rows of ") + name +
                                    " must begin at multiples of 16 bytes");
    if ((t.size(0) - 1) * ld + wide + t.storage_offset() > (int64_t)t.storage().nbytes())
        throw std::invalid_argument(std::string("the last row of ") + name +
                                    " must be allocated up to a multiple of 16 bytes");
    return ld;
}
Tensor empty(at::IntArrayRef shape, at::ScalarType type, const Tensor &ref) {
    return at::empty(shape, at::TensorOptions().dtype(type).device(ref.device()));
}
// Nothing is recorded for autograd, so a gradient that someone waits for would
// be lost without a word.
bool wants_grad(const Tensor &t) { return t.defined() && t.requires_grad(); }
bool wants_grad(const Maybe &t) { return t && wants_grad(*t); }
template <typename... Ts> void no_grad(const Ts &...t) {
    need(!at::GradMode::is_enabled() || !(wants_grad(t) || ...),
         "a tensor requires grad, and the operators record nothing for autograd: detach it or "
         "call under torch.no_grad()");
}
// Given outputs have changed: what autograd saved of them is stale.
void wrote(const Tensor &t) {
    if (t.defined() && !t.is_inference()) t.unsafeGetTensorImpl()->bump_version();
}
void wrote(const Maybe &t) {
    if (t && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}
// Device scratch of a call on the current stream.
void *scratch(size_t bytes, Tensor &keep, const Tensor &ref) {
    if (!bytes) return nullptr;
    keep = empty({(int64_t)bytes}, at::kByte, ref);
    return keep.data_ptr();
}

// ------------------------------------------------------------- group norm

struct Map { int32_t n, c; int64_t hw; };
Map map_of(const Tensor &x, int64_t groups) {
    on_gpu(x, "x");
    need(real_type(x), "x must be float32, float16 or bfloat16");
    need(x.dim() >= 2 && x.is_contiguous(), "x must be a contiguous [n, ..., c] map");
    const int64_t c = x.size(-1), n = x.size(0);
    need(groups >= 1 && c >= 1 && c % groups == 0, "groups do not divide the channels");
    int64_t hw = 1;
    for (int64_t d = 1; d + 1 < x.dim(); d++) hw *= x.size(d);
    need(hw >= 1, "x has no pixels");
    need(n < (int64_t)1 << 31 && c < (int64_t)1 << 31, "x is too large");
    return Map{(int32_t)n, (int32_t)c, hw};
}
size_t norm_bytes(const Tensor &x, const Map &m, int64_t groups, bool backward) {
    size_t b = 0;
    done(ctc_group_norm_workspace_bytes(code(x), m.n, m.hw, m.c, (int32_t)groups, backward, &b));
    return b;
}

std::tuple<Tensor, Tensor, Tensor> group_norm(const Tensor &x, int64_t groups, const Maybe &gamma,
                                              const Maybe &beta, const Maybe &residual, int act,
                                              bool carry, double eps, Maybe y, Maybe mean,
                                              Maybe rstd, int64_t stream) {
    const Map m = map_of(x, groups);
    no_grad(x, gamma, beta, residual, y, mean, rstd);
    c10::DeviceGuard guard(x.device());
    if (!y) {
        y = at::empty_like(x);
        const Tensor stats = empty({2, m.n, groups}, at::kFloat, x);
        mean = stats[0];
        rstd = stats[1];
    }
    need(mean && rstd, "out must hold y, mean and rstd");
    const std::array<int64_t, 1> per_c{m.c};
    const std::array<int64_t, 2> per_g{m.n, groups};
    void *g = like(gamma, "gamma", at::kFloat, per_c, x), *b = like(beta, "beta", at::kFloat, per_c, x);
    void *r = like(residual, "residual", x), *yp = like(y, "y", x);
    void *mp = like(mean, "mean", at::kFloat, per_g, x), *rp = like(rstd, "rstd", at::kFloat, per_g, x);
    Tensor keep;
    const size_t bytes = norm_bytes(x, m, groups, false);
    done(ctc_group_norm_forward(code(x), m.n, m.hw, m.c, (int32_t)groups, carry, x.data_ptr(),
                                (float *)g, (float *)b, r, (float)eps, act, yp, (float *)mp,
                                (float *)rp, scratch(bytes, keep, x), bytes, (void *)stream));
    for (const Maybe *t : {&y, &mean, &rstd}) wrote(*t);
    return {*y, *mean, *rstd};
}

std::tuple<Maybe, Maybe, Maybe, Maybe>
group_norm_backward(const Tensor &dy, const Tensor &x, const Tensor &mean, const Tensor &rstd,
                    int64_t groups, const Maybe &gamma, const Maybe &beta, const Maybe &residual,
                    int act, bool carry, bool make, Maybe dx, Maybe dr, Maybe dgamma, Maybe dbeta,
                    int64_t stream) {
    const Map m = map_of(x, groups);
    no_grad(dy, x, mean, rstd, gamma, beta, residual, dx, dr, dgamma, dbeta);
    c10::DeviceGuard guard(x.device());
    if (make) {
        dx = at::empty_like(x);
        if (residual) dr = at::empty_like(x);
        const Tensor both = empty({2, m.c}, at::kFloat, x);
        dgamma = both[0];
        dbeta = both[1];
    }
    need(!dx || !dr || m.n == 0 || dx->data_ptr() != dr->data_ptr(),
         "dx and dresidual must differ");
    const std::array<int64_t, 1> per_c{m.c};
    const std::array<int64_t, 2> per_g{m.n, groups};
    void *dyp = like(dy, "dy", x), *mp = like(mean, "mean", at::kFloat, per_g, x);
    void *rp = like(rstd, "rstd", at::kFloat, per_g, x);
    void *g = like(gamma, "gamma", at::kFloat, per_c, x), *b = like(beta, "beta", at::kFloat, per_c, x);
    void *r = like(residual, "residual", x);
    void *dxp = like(dx, "dx", x), *drp = like(dr, "dresidual", x);
    void *dg = like(dgamma, "dgamma", at::kFloat, per_c, x);
    void *db = like(dbeta, "dbeta", at::kFloat, per_c, x);
    Tensor keep;
    const size_t bytes = norm_bytes(x, m, groups, true);
    done(ctc_group_norm_backward(code(x), m.n, m.hw, m.c, (int32_t)groups, carry, dyp,
                                 x.data_ptr(), (float *)mp, (float *)rp, (float *)g, (float *)b, r,
                                 act, dxp, drp, (float *)dg, (float *)db,
                                 scratch(bytes, keep, x), bytes, (void *)stream));
    for (const Maybe *t : {&dx, &dr, &dgamma, &dbeta}) wrote(*t);
    return {dx, dr, dgamma, dbeta};
}

// --------------------------------------------------------- 8-bit matrices

std::tuple<Tensor, Tensor> fp8_quantize(const Tensor &x, bool e5m2, int64_t block, bool transpose,
                                        Maybe q, Maybe scales, int64_t stream) {
    on_gpu(x, "x");
    need(real_type(x), "x must be float32, float16 or bfloat16");
    need(block == 1 || block == 128, "block_rows must be 1 or 128");
    no_grad(x, q, scales);
    const int64_t ldx = rows_of(x, "x", x);
    const int64_t rows = x.size(0), cols = x.size(1);
    const int64_t qr = transpose ? cols : rows, qc = transpose ? rows : cols;
    const std::array<int64_t, 2> shape{(qc + 127) / 128, (qr + block - 1) / block};
    const at::ScalarType type = e5m2 ? at::kFloat8_e5m2 : at::kFloat8_e4m3fn;
    c10::DeviceGuard guard(x.device());
    if (!q) {
        const int64_t ld = (qc + 15) / 16 * 16;
        q = empty({qr, ld}, type, x);
        if (ld != qc) q = q->slice(1, 0, qc);
        scales = empty(shape, at::kFloat, x);
    }
    need(scales.has_value(), "out must hold q and scales");
    need(q->scalar_type() == type && q->dim() == 2 && q->size(0) == qr && q->size(1) == qc,
         "q must be a " + std::string(c10::toString(type)) + " matrix of shape [" +
             std::to_string(qr) + ", " + std::to_string(qc) + "]");
    const int64_t ldq = rows_8bit(*q, "q", x);
    void *sp = like(scales, "scales", at::kFloat, shape, x);
    done(ctc_fp8_quantize(code(x), rows, cols, x.data_ptr(), ldx, code(*q), (int32_t)block,
                          transpose, q->data_ptr(), ldq, (float *)sp, shape[1], (void *)stream));
    wrote(q);
    wrote(scales);
    return {*q, *scales};
}

int32_t scale_rows(const Tensor &s, const char *name, int64_t rows, int64_t kb, const Tensor &ref) {
    const int64_t rb = (rows + 127) / 128;
    if (s.scalar_type() != at::kFloat || s.dim() != 2 || s.device() != ref.device() ||
        !s.is_contiguous() || s.size(0) != kb || (s.size(1) != rows && s.size(1) != rb))
        throw std::invalid_argument(std::string(name) +
                                    " must be a contiguous float32 tensor of shape (" +
                                    std::to_string(kb) + ", " + std::to_string(rows) + ") or (" +
                                    std::to_string(kb) + ", " + std::to_string(rb) + ") on " +
                                    ref.device().str());
    return s.size(1) == rows ? 1 : 128;
}

Tensor fp8_matmul(const Tensor &a, const Tensor &a_scales, const Tensor &b,
                  const Tensor &b_scales, const Maybe &bias, int act, at::ScalarType dtype,
                  const Maybe &out, int64_t stream) {
    on_gpu(a, "a");
    need(byte_type(a) && byte_type(b), "a and b must be float8 tensors");
    no_grad(a, a_scales, b, b_scales, bias, out);
    const int64_t lda = rows_8bit(a, "a", a), ldb = rows_8bit(b, "b", a);
    const int64_t m = a.size(0), k = a.size(1), n = b.size(0), kb = (k + 127) / 128;
    need(b.size(1) == k, "a and b must have the same number of columns");
    const int32_t ab = scale_rows(a_scales, "a_scales", m, kb, a);
    const int32_t bb = scale_rows(b_scales, "b_scales", n, kb, a);
    c10::DeviceGuard guard(a.device());
    need(out || dtype == at::kFloat || dtype == at::kHalf || dtype == at::kBFloat16,
         "dtype must be float32, float16 or bfloat16");
    const Tensor y = out ? *out : empty({m, n}, dtype, a);
    need(real_type(y) && y.dim() == 2 && y.size(0) == m && y.size(1) == n,
         "out must be a float32, float16 or bfloat16 matrix of shape [" + std::to_string(m) +
             ", " + std::to_string(n) + "]");
    const int64_t ldy = rows_of(y, "out", a);
    void *bp = like(bias, "bias", at::kFloat, std::array<int64_t, 1>{n}, a);
    Tensor keep;
    size_t bytes = 0;
    done(ctc_fp8_matmul_workspace_bytes(code(y), m, n, k, bb, &bytes));
    done(ctc_fp8_matmul(code(a), code(b), code(y), m, n, k, a.data_ptr(), lda,
                        a_scales.data_ptr<float>(), a_scales.size(1), ab, b.data_ptr(), ldb,
                        b_scales.data_ptr<float>(), b_scales.size(1), bb, (float *)bp, act,
                        y.data_ptr(), ldy, scratch(bytes, keep, a), bytes, (void *)stream));
    wrote(out);
    return y;
}

// ----------------------------------------------------------------- scores

int64_t logits_of(const Tensor &x) {
    on_gpu(x, "logits");
    need(real_type(x), "logits must be float32, float16 or bfloat16");
    const int64_t ld = rows_of(x, "logits", x);
    need(x.size(1) >= 1, "logits without columns");
    need(x.size(1) < (int64_t)1 << 31, "too many columns");
    return ld;
}

// lse, entropy, logprob, rank, top_ids, top_logprobs
typedef std::tuple<Maybe, Maybe, Maybe, Maybe, Maybe, Maybe> Scores;
Scores token_scores(const Tensor &x, const Maybe &targets, int64_t top_k, bool make, Scores out,
                    int64_t stream) {
    const int64_t ld = logits_of(x), rows = x.size(0);
    const int32_t vocab = (int32_t)x.size(1);
    c10::DeviceGuard guard(x.device());
    auto &[lse, entropy, logprob, rank, ids, tops] = out;
    no_grad(x, lse, entropy, logprob, tops);
    if (make) {
        const Tensor f = empty({targets ? 3 : 2, rows}, at::kFloat, x);
        lse = f[0];
        entropy = f[1];
        if (targets) {
            logprob = f[2];
            rank = empty({rows}, at::kInt, x);
        }
        if (top_k > 0) {
            ids = empty({rows, top_k}, at::kInt, x);
            tops = empty({rows, top_k}, at::kFloat, x);
        }
    }
    const std::array<int64_t, 1> per{rows};
    const std::array<int64_t, 2> best{rows, top_k};
    void *tp = like(targets, "targets", at::kInt, per, x);
    void *lp = like(lse, "lse", at::kFloat, per, x), *pp = like(logprob, "logprob", at::kFloat, per, x);
    void *ep = like(entropy, "entropy", at::kFloat, per, x), *rp = like(rank, "rank", at::kInt, per, x);
    void *ip = like(ids, "top_ids", at::kInt, best, x);
    void *vp = like(tops, "top_logprobs", at::kFloat, best, x);
    size_t bytes = 0;
    Tensor keep;
    done(ctc_token_scores_workspace_bytes(rows, vocab, (int32_t)top_k, &bytes));
    done(ctc_token_scores_forward(code(x), rows, vocab, x.data_ptr(), ld, (int32_t *)tp,
                                  (int32_t)top_k, (float *)lp, (float *)pp, (float *)ep,
                                  (int32_t *)rp, (int32_t *)ip, (float *)vp,
                                  scratch(bytes, keep, x), bytes, (void *)stream));
    for (const Maybe *t : {&lse, &entropy, &logprob, &rank, &ids, &tops}) wrote(*t);
    return out;
}

Tensor token_scores_backward(const Tensor &x, const Maybe &targets, const Tensor &lse,
                             const Maybe &entropy, const Maybe &g_lse, const Maybe &g_logprob,
                             const Maybe &g_entropy, const Maybe &out, int64_t stream) {
    const int64_t ld = logits_of(x), rows = x.size(0);
    no_grad(x, lse, entropy, g_lse, g_logprob, g_entropy, out);
    c10::DeviceGuard guard(x.device());
    const Tensor dx = out ? *out : empty({rows, x.size(1)}, x.scalar_type(), x);
    need(dx.scalar_type() == x.scalar_type() && dx.sizes() == x.sizes(), "out must be like logits");
    const int64_t ldd = rows_of(dx, "out", x);
    const std::array<int64_t, 1> per{rows};
    void *tp = like(targets, "targets", at::kInt, per, x), *lp = like(lse, "lse", at::kFloat, per, x);
    void *ep = like(entropy, "entropy", at::kFloat, per, x);
    void *gl = like(g_lse, "g_lse", at::kFloat, per, x);
    void *gp = like(g_logprob, "g_logprob", at::kFloat, per, x);
    void *ge = like(g_entropy, "g_entropy", at::kFloat, per, x);
    done(ctc_token_scores_backward(code(x), rows, (int32_t)x.size(1), x.data_ptr(), ld,
                                   (int32_t *)tp, (float *)lp, (float *)ep, (float *)gl,
                                   (float *)gp, (float *)ge, dx.data_ptr(), ldd, (void *)stream));
    wrote(out);
    return dx;
}

// -------------------------------------------------------------- attention

// A tensor [batch, tokens, heads, head] of that shape and type whose heads are
// contiguous.
ctc_heads heads_of(const Tensor &t, const char *name, const std::array<int64_t, 4> &shape,
                   at::ScalarType type, const Tensor &ref) {
    if (!t.defined() || t.scalar_type() != type || t.sizes() != at::IntArrayRef(shape) ||
        t.device() != ref.device())
        throw std::invalid_argument(std::string(name) + " must be a tensor of type " +
                                    c10::toString(type) + " and shape " +
                                    c10::str(at::IntArrayRef(shape)) + " on " +
                                    ref.device().str());
    if (shape[3] > 1 && t.stride(3) != 1)
        throw std::invalid_argument(std::string("the heads of ") + name + " must be contiguous");
    return ctc_heads{t.data_ptr(), {t.stride(0), t.stride(1), t.stride(2)}};
}
const int32_t *lengths_of(const Maybe &t, const char *name, int64_t b, const Tensor &ref) {
    return (const int32_t *)like(t, name, at::kInt, std::array<int64_t, 1>{b}, ref);
}
bool small(int64_t v) { return v < (int64_t)1 << 31; }

struct Attention {
    ctc_attention a;
    std::array<int64_t, 4> qs, ks;
    ctc_heads q, k, v;
    size_t bytes = 0;
    Attention(const Tensor &tq, const Tensor &tk, const Tensor &tv, bool causal,
              const Maybe &q_lengths, const Maybe &k_lengths, const std::optional<double> &scale,
              bool backward) {
        on_gpu(tq, "q");
        need(tq.scalar_type() == at::kHalf || tq.scalar_type() == at::kBFloat16,
             "q must be float16 or bfloat16");
        need(tq.dim() == 4 && tk.dim() == 4, "q and k must be [batch, tokens, heads, head size]");
        for (int i = 0; i < 4; i++)
            need(small(tq.size(i)) && small(tk.size(i)), "q or k is too large");
        const int64_t d = tq.size(3);
        qs = {tq.size(0), tq.size(1), tq.size(2), d};
        ks = {qs[0], tk.size(1), tk.size(2), d};
        q = heads_of(tq, "q", qs, tq.scalar_type(), tq);
        k = heads_of(tk, "k", ks, tq.scalar_type(), tq);
        v = heads_of(tv, "v", ks, tq.scalar_type(), tq);
        need(d >= 1, "heads without values");
        a = ctc_attention{};
        a.dtype = code(tq);
        a.batch = (int32_t)qs[0];
        a.queries = (int32_t)qs[1];
        a.keys = (int32_t)ks[1];
        a.q_heads = (int32_t)qs[2];
        a.k_heads = (int32_t)ks[2];
        a.head = (int32_t)d;
        a.causal = causal;
        a.scale = scale ? (float)*scale : 1.f / std::sqrt((float)d);
        a.q_lengths = lengths_of(q_lengths, "q_lengths", qs[0], tq);
        a.k_lengths = lengths_of(k_lengths, "k_lengths", qs[0], tq);
        done(ctc_attention_workspace_bytes(&a, backward, &bytes));
    }
};

std::tuple<Tensor, Tensor> attention(const Tensor &q, const Tensor &k, const Tensor &v,
                                     bool causal, const Maybe &q_lengths, const Maybe &k_lengths,
                                     const std::optional<double> &scale, Maybe o, Maybe lse,
                                     int64_t stream) {
    const Attention c(q, k, v, causal, q_lengths, k_lengths, scale, false);
    no_grad(q, k, v, o, lse);
    c10::DeviceGuard guard(q.device());
    const std::array<int64_t, 3> rows{c.qs[0], c.qs[2], c.qs[1]};
    if (!o) {
        o = empty(c.qs, q.scalar_type(), q);
        lse = empty(rows, at::kFloat, q);
    }
    need(lse.has_value(), "out must hold o and lse");
    const ctc_heads oh = heads_of(*o, "o", c.qs, q.scalar_type(), q);
    void *lp = like(lse, "lse", at::kFloat, rows, q);
    Tensor keep;
    done(ctc_attention_forward(&c.a, &c.q, &c.k, &c.v, &oh, (float *)lp,
                               scratch(c.bytes, keep, q), c.bytes, (void *)stream));
    wrote(o);
    wrote(lse);
    return {*o, *lse};
}

std::tuple<Tensor, Tensor, Tensor>
attention_backward(const Tensor &dout, const Tensor &q, const Tensor &k, const Tensor &v,
                   const Tensor &o, const Tensor &lse, bool causal, const Maybe &q_lengths,
                   const Maybe &k_lengths, const std::optional<double> &scale, Maybe dq, Maybe dk,
                   Maybe dv, int64_t stream) {
    const Attention c(q, k, v, causal, q_lengths, k_lengths, scale, true);
    no_grad(dout, q, k, v, o, lse, dq, dk, dv);
    c10::DeviceGuard guard(q.device());
    const at::ScalarType type = q.scalar_type();
    if (!dq) {
        dq = empty(c.qs, type, q);
        dk = empty(c.ks, type, q);
        dv = empty(c.ks, type, q);
    }
    need(dk && dv, "out must hold dq, dk and dv");
    const ctc_heads doh = heads_of(dout, "do", c.qs, type, q), oh = heads_of(o, "o", c.qs, type, q);
    const ctc_heads dqh = heads_of(*dq, "dq", c.qs, type, q);
    const ctc_heads dkh = heads_of(*dk, "dk", c.ks, type, q);
    const ctc_heads dvh = heads_of(*dv, "dv", c.ks, type, q);
    void *lp = like(lse, "lse", at::kFloat, std::array<int64_t, 3>{c.qs[0], c.qs[2], c.qs[1]}, q);
    Tensor keep;
    done(ctc_attention_backward(&c.a, &doh, &c.q, &c.k, &c.v, &oh, (float *)lp, &dqh, &dkh, &dvh,
                                scratch(c.bytes, keep, q), c.bytes, (void *)stream));
    for (const Maybe *t : {&dq, &dk, &dv}) wrote(*t);
    return {*dq, *dk, *dv};
}

// ------------------------------------------------------------- head norms

struct HeadNorm {
    ctc_head_rotary h;
    std::array<int64_t, 4> qs, ks;
    ctc_heads q, k;
    HeadNorm(const Tensor &tq, const Maybe &tk, const Maybe &qw, const Maybe &kw,
             const Maybe &positions, const Maybe &frequencies, const std::vector<int64_t> &axes,
             bool interleaved, bool norm, double eps, at::ScalarType out) {
        on_gpu(tq, "q");
        need(real_type(tq), "q must be float32, float16 or bfloat16");
        need(out == tq.scalar_type() || (tq.scalar_type() == at::kFloat &&
                                         (out == at::kHalf || out == at::kBFloat16)),
             "dtype must be q's, or a narrower one for float32");
        need(tq.dim() == 4 && (!tk || tk->dim() == 4),
             "q and k must be [batch, tokens, heads, head size]");
        need(axes.size() <= 4, "up to 4 position axes");
        for (int i = 0; i < 4; i++)
            need(small(tq.size(i)) && (!tk || small(tk->size(i))), "q or k is too large");
        qs = {tq.size(0), tq.size(1), tq.size(2), tq.size(3)};
        ks = {qs[0], qs[1], tk ? tk->size(2) : 0, qs[3]};
        need(qs[3] >= 2 && qs[2] >= 1, "q without heads or values");
        h = ctc_head_rotary{};
        q = heads_of(tq, "q", qs, tq.scalar_type(), tq);
        k = tk ? heads_of(*tk, "k", ks, tq.scalar_type(), tq) : ctc_heads{};
        h.dtype = code(tq);
        h.ytype = out == at::kFloat ? CTC_F32 : out == at::kHalf ? CTC_F16 : CTC_BF16;
        h.batch = (int32_t)qs[0];
        h.tokens = (int32_t)qs[1];
        h.q_heads = (int32_t)qs[2];
        h.k_heads = (int32_t)ks[2];
        h.head = (int32_t)qs[3];
        h.norm = norm;
        h.eps = (float)eps;
        h.interleaved = interleaved;
        const std::array<int64_t, 1> per{qs[3]};
        h.q_weight = (const float *)like(qw, "q_weight", at::kFloat, per, tq);
        h.k_weight = (const float *)like(kw, "k_weight", at::kFloat, per, tq);
        h.axes = (int32_t)axes.size();
        int64_t turned = 0;
        for (size_t i = 0; i < axes.size(); i++) {
            need(axes[i] >= 0 && axes[i] <= qs[3] / 2, "bad pairs of an axis");
            h.pairs[i] = (int32_t)axes[i];
            turned += axes[i];
        }
        need(axes.empty() || (positions && frequencies), "axes need positions and frequencies");
        if (axes.empty()) return;
        const int64_t n = (int64_t)axes.size();
        h.per_image = positions->dim() == 3;
        h.positions = (const int32_t *)(
            h.per_image ? like(positions, "positions", at::kInt,
                               std::array<int64_t, 3>{qs[0], qs[1], n}, tq)
                        : like(positions, "positions", at::kInt,
                               std::array<int64_t, 2>{qs[1], n}, tq));
        h.frequencies = (const float *)like(frequencies, "frequencies", at::kFloat,
                                            std::array<int64_t, 1>{turned}, tq);
    }
};

std::tuple<Tensor, Maybe> head_norm_rotary(const Tensor &q, const Maybe &k, const Maybe &qw,
                                           const Maybe &kw, const Maybe &positions,
                                           const Maybe &frequencies,
                                           const std::vector<int64_t> &axes, bool interleaved,
                                           bool norm, double eps,
                                           const std::optional<at::ScalarType> &dtype, Maybe yq,
                                           Maybe yk, int64_t stream) {
    const at::ScalarType type = yq ? yq->scalar_type() : dtype ? *dtype : q.scalar_type();
    const HeadNorm c(q, k, qw, kw, positions, frequencies, axes, interleaved, norm, eps, type);
    no_grad(q, k, qw, kw, frequencies, yq, yk);
    c10::DeviceGuard guard(q.device());
    if (!yq) {
        yq = empty(c.qs, type, q);
        if (k) yk = empty(c.ks, type, q);
    }
    need(!k || yk, "out must hold both results");
    const ctc_heads qh = heads_of(*yq, "out", c.qs, type, q);
    const ctc_heads kh = k ? heads_of(*yk, "out", c.ks, type, q) : ctc_heads{};
    done(ctc_head_norm_rotary_forward(&c.h, &c.q, &c.k, &qh, &kh, (void *)stream));
    wrote(yq);
    if (k) wrote(yk);
    return {*yq, k ? yk : Maybe()};
}

std::tuple<Tensor, Maybe, Maybe, Maybe>
head_norm_rotary_backward(const Tensor &dyq, const Maybe &dyk, const Tensor &q, const Maybe &k,
                          const Maybe &qw, const Maybe &kw, const Maybe &positions,
                          const Maybe &frequencies, const std::vector<int64_t> &axes,
                          bool interleaved, bool norm, double eps, bool make, Maybe dq, Maybe dk,
                          Maybe dqw, Maybe dkw, int64_t stream) {
    need(dyq.defined(), "dq must be a tensor");
    const at::ScalarType type = dyq.scalar_type();
    const HeadNorm c(q, k, qw, kw, positions, frequencies, axes, interleaved, norm, eps, type);
    no_grad(dyq, dyk, q, k, qw, kw, frequencies, dq, dk, dqw, dkw);
    need(!k || dyk, "the gradient of the keys is needed");
    c10::DeviceGuard guard(q.device());
    if (make) {
        dq = empty(c.qs, q.scalar_type(), q);
        const Tensor both = empty({2, c.qs[3]}, at::kFloat, q);
        dqw = both[0];
        if (k) {
            dk = empty(c.ks, q.scalar_type(), q);
            dkw = both[1];
        }
    }
    need(dq && (!k || dk), "out must hold the gradients of q and k");
    const ctc_heads dyqh = heads_of(dyq, "dq", c.qs, type, q);
    const ctc_heads dykh = k ? heads_of(*dyk, "dk", c.ks, type, q) : ctc_heads{};
    const ctc_heads dqh = heads_of(*dq, "out", c.qs, q.scalar_type(), q);
    const ctc_heads dkh = k ? heads_of(*dk, "out", c.ks, q.scalar_type(), q) : ctc_heads{};
    const std::array<int64_t, 1> per{c.qs[3]};
    void *qwp = like(dqw, "the gradient of q_weight", at::kFloat, per, q);
    void *kwp = k ? like(dkw, "the gradient of k_weight", at::kFloat, per, q) : nullptr;
    size_t bytes = 0;
    Tensor keep;
    done(ctc_head_norm_rotary_workspace_bytes(&c.h, &bytes));
    done(ctc_head_norm_rotary_backward(&c.h, &dyqh, &dykh, &c.q, &c.k, &dqh, &dkh, (float *)qwp,
                                       (float *)kwp, scratch(bytes, keep, q), bytes,
                                       (void *)stream));
    wrote(dq);
    wrote(dqw);
    if (k) {
        wrote(dk);
        wrote(dkw);
    }
    return {*dq, k ? dk : Maybe(), dqw, k ? dkw : Maybe()};
}

// --------------------------------------------------------------- clipping

// The tensors of a list or tuple, as long as `held` lives.  (pybind11's own
// conversion asks each for its class and counts references: 0.1 us a tensor.)
std::vector<const Tensor *> tensors_of(const py::object &list, py::object &held) {
    held = py::reinterpret_steal<py::object>(
        PySequence_Fast(list.ptr(), "a list or tuple of tensors is needed"));
    if (!held) throw py::error_already_set();
    std::vector<const Tensor *> r(PySequence_Fast_GET_SIZE(held.ptr()));
    for (size_t i = 0; i < r.size(); i++) {
        PyObject *o = PySequence_Fast_GET_ITEM(held.ptr(), i);
        need((PyObject *)Py_TYPE(o) == THPVariableClass || THPVariable_Check(o),
             "a list or tuple of tensors is needed");
        r[i] = &THPVariable_Unpack(o);
    }
    return r;
}
// (the norm, and the outputs where they are made here: a list that the caller
// holds need not become one again)
std::tuple<Tensor, std::optional<std::vector<Tensor>>>
clip_gradients(const py::object &grad_list, double max_norm, const py::object &out_list,
               bool in_place, Maybe norm, int64_t stream) {
    py::object held, held_out;
    const std::vector<const Tensor *> grads = tensors_of(grad_list, held);
    std::vector<const Tensor *> out;
    const bool given_out = !out_list.is_none();
    if (given_out) out = tensors_of(out_list, held_out);
    need(!grads.empty(), "no gradients");
    const Tensor &ref = *grads[0];
    on_gpu(ref, "a gradient");
    c10::DeviceGuard guard(ref.device());
    need(!given_out || out.size() == grads.size(), "out must hold a tensor for each gradient");
    std::vector<ctc_gradient> g(grads.size());
    std::optional<std::vector<Tensor>> made;
    if (!given_out && !in_place) {
        made.emplace();
        made->reserve(grads.size());
    }
    for (size_t i = 0; i < grads.size(); i++) {
        const Tensor &x = *grads[i];
        need(x.defined() && real_type(x) && x.device() == ref.device(),
             "gradients must be float32, float16 or bfloat16 tensors of one GPU");
        need(x.is_contiguous() || x.is_non_overlapping_and_dense(), "gradients must be dense");
        no_grad(x);
        if (made) made->push_back(at::empty_like(x));
        const Tensor &y = made ? (*made)[i] : given_out ? *out[i] : x;
        if (given_out) {
            no_grad(y);
            need(y.defined() && y.scalar_type() == x.scalar_type() && y.device() == x.device() &&
                     y.sizes() == x.sizes() && ((y.is_contiguous() && x.is_contiguous()) ||
                                                y.strides() == x.strides()),
                 "out must be like the gradients");
        }
        g[i] = ctc_gradient{x.data_ptr(), y.data_ptr(), x.numel(), (int32_t)code(x), 0};
    }
    const bool given = norm.has_value();
    if (!given) norm = empty({}, at::kFloat, ref);
    need(norm->scalar_type() == at::kFloat && norm->numel() == 1 && norm->device() == ref.device(),
         "the norm must be one float32 value");
    size_t bytes = 0;
    Tensor keep;
    done(ctc_clip_gradients_workspace_bytes((int32_t)g.size(), g.data(), &bytes));
    done(ctc_clip_gradients_to((int32_t)g.size(), g.data(), max_norm, (float *)norm->data_ptr(),
                               scratch(bytes, keep, ref), bytes, (void *)stream));
    if (!made)
        for (const Tensor *t : given_out ? out : grads) wrote(*t);
    if (given) wrote(norm);
    return {*norm, made};
}

}  // namespace

PYBIND11_MODULE(_binding, m) {
    m.def("set_check", [](py::object f) { check_status = std::move(f); });
    m.def("group_norm", &group_norm);
    m.def("group_norm_backward", &group_norm_backward);
    m.def("fp8_quantize", &fp8_quantize);
    m.def("fp8_matmul", &fp8_matmul);
    m.def("token_scores", &token_scores);
    m.def("token_scores_backward", &token_scores_backward);
    m.def("attention", &attention);
    m.def("attention_backward", &attention_backward);
    m.def("head_norm_rotary", &head_norm_rotary);
    m.def("head_norm_rotary_backward", &head_norm_rotary_backward);
    m.def("clip_gradients", &clip_gradients);
    m.add_object("_cleanup", py::capsule([]() { check_status.release(); }));
}
