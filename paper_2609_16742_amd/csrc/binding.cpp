// Python binding of the operators around a protected classifier: checks
// torch tensors, allocates outputs and workspaces, calls the C ABI
// (include/ctc.h).  Marshalling only, compiled because an operator on a
// small batch runs for five microseconds and the same checks in Python took
// ten.  No torch types cross the C ABI: this is its caller.
#include <torch/csrc/utils/pybind.h>

#include <ATen/ATen.h>
#include <ATen/core/grad_mode.h>

#include <optional>
#include <stdexcept>
#include <string>
#include <tuple>

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

}  // namespace

PYBIND11_MODULE(_binding, m) {
    m.def("set_check", [](py::object f) { check_status = std::move(f); });
    m.def("group_norm", &group_norm);
    m.def("group_norm_backward", &group_norm_backward);
    m.def("fp8_quantize", &fp8_quantize);
    m.def("fp8_matmul", &fp8_matmul);
    m.def("token_scores", &token_scores);
    m.def("token_scores_backward", &token_scores_backward);
    m.add_object("_cleanup", py::capsule([]() { check_status.release(); }));
}
