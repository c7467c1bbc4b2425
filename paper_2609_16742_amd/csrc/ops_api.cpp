// C ABI of the operators around a protected classifier (include/ctc.h):
// checks the arguments, then enqueues the kernels of ops.hip.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <exception>
#include <numeric>
#include <vector>

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

// -------------------------------------------------------------- attention

// Strides of a tensor of heads, those of dimensions of size 1 as 0.
void heads_strides(const ctc_heads &h, const int64_t (&size)[3], int64_t (&out)[3]) {
    for (int i = 0; i < 3; i++) out[i] = size[i] > 1 ? h.strides[i] : 0;
}
// Address and strides of a tensor of heads.  Outputs must not overlap
// themselves: each stride reaches past what smaller ones span.
ctc_status heads_arg(const ctc_heads *h, const char *name, int64_t b, int64_t t, int64_t heads,
                     int64_t d, bool out, const void *&data, int64_t (&strides)[3]) {
    data = nullptr;
    for (int64_t &v : strides) v = 0;
    if (!(b && t && heads)) return CTC_OK;
    if (!h || !h->data) return fail(CTC_ERR_ARG, "NULL %s", name);
    const int64_t size[3] = {b, t, heads};
    heads_strides(*h, size, strides);
    for (int64_t v : strides)
        if (v < 0 || v > (int64_t)1 << 45) return fail(CTC_ERR_ARG, "bad strides of %s", name);
    if (out) {
        int64_t span = d;
        bool done[3] = {false, false, false};
        for (int n = 0; n < 3; n++) {
            int best = -1;
            for (int i = 0; i < 3; i++)
                if (!done[i] && size[i] > 1 && (best < 0 || strides[i] < strides[best])) best = i;
            if (best < 0) break;
            if (strides[best] < span) return fail(CTC_ERR_ARG, "elements of %s overlap", name);
            span += (size[best] - 1) * strides[best];
            done[best] = true;
        }
    }
    data = h->data;
    return CTC_OK;
}

// Elements of a tensor of heads (or, as one head, of a dense one), in bytes:
// runs of `run` bytes at three strides.
struct Region {
    uintptr_t at = 0;
    int64_t size[3] = {0, 0, 0}, stride[3] = {0, 0, 0}, run = 0;
    bool empty() const { return !run || !size[0] || !size[1] || !size[2]; }
    double end() const {
        double e = (double)at + (double)run;
        for (int i = 0; i < 3; i++) e += (double)(size[i] - 1) * (double)stride[i];
        return e;
    }
    bool operator==(const Region &o) const {
        return at == o.at && run == o.run && std::equal(size, size + 3, o.size) &&
               std::equal(stride, stride + 3, o.stride);
    }
};
Region region(const void *data, int64_t b, int64_t t, int64_t heads, const int64_t (&strides)[3],
              int64_t d, int type) {
    Region r;
    const int64_t bytes = type_bytes(type), size[3] = {b, t, heads};
    r.at = (uintptr_t)data;
    r.run = data ? d * bytes : 0;
    for (int i = 0; i < 3; i++) {
        r.size[i] = size[i];
        r.stride[i] = strides[i] * bytes;
    }
    return r;
}
Region dense(const void *data, int64_t n, int type) {
    return region(data, 1, 1, 1, {0, 0, 0}, n, type);
}
// Whether a byte is of both.  Parts of one buffer may lie within each other's
// span, so what is looked for is a run of each, at whole multiples of their
// strides, that meet: multiples of equal strides count as one, strides are gone
// through from the largest down, and only where what the smaller ones reach can
// still close the gap, which for such parts leaves one or two choices each.
struct Meeting {
    struct Step { int64_t stride, lo, hi; };
    Step step[6];
    int64_t lo[7], hi[7];                        // reach of the steps from i on
    int n = 0, left = 1 << 16;
    void add(int64_t stride, int64_t from, int64_t to) {
        for (int i = 0; i < n; i++)
            if (step[i].stride == stride) {
                step[i].lo += from;
                step[i].hi += to;
                return;
            }
        if (stride && from < to) step[n++] = Step{stride, from, to};
    }
    static int64_t over(int64_t a, int64_t b) { return a / b - (a % b < 0); }   // rounded down
    // a sum of multiples of the steps from i on within from .. to
    bool find(int i, int64_t from, int64_t to) {
        if (to < lo[i] || from > hi[i]) return false;
        if (i == n) return true;
        // (choices beyond any that parts of a buffer leave: not told apart)
        if (--left < 0) return true;
        const Step &s = step[i];
        int64_t a = -over(hi[i + 1] - from, s.stride), b = over(to - lo[i + 1], s.stride);
        if (a < s.lo) a = s.lo;
        if (b > s.hi) b = s.hi;
        if (b - a > 8) {
            int64_t g = 0;
            for (int k = i; k < n; k++) g = std::gcd(g, step[k].stride);
            if (over(to, g) * g < from) return false;
        }
        for (int64_t v = a; v <= b; v++)
            if (find(i + 1, from - v * s.stride, to - v * s.stride)) return true;
        return false;
    }
    bool of(const Region &a, const Region &b) {
        for (int i = 0; i < 3; i++) {
            add(a.stride[i], 0, a.size[i] - 1);
            add(b.stride[i], 1 - b.size[i], 0);
        }
        std::sort(step, step + n, [](const Step &x, const Step &y) { return x.stride > y.stride; });
        lo[n] = hi[n] = 0;
        for (int i = n - 1; i >= 0; i--) {
            lo[i] = lo[i + 1] + step[i].lo * step[i].stride;
            hi[i] = hi[i + 1] + step[i].hi * step[i].stride;
        }
        const int64_t gap = (int64_t)(b.at - a.at);
        return find(0, gap - (a.run - 1), gap + (b.run - 1));
    }
};
bool meet(const Region &a, const Region &b) {
    if (a.empty() || b.empty()) return false;
    const double x = a.end(), y = b.end();
    if (x <= (double)b.at || y <= (double)a.at) return false;
    // (no memory is that long)
    if (x >= 0x1p61 || y >= 0x1p61) return true;
    return Meeting().of(a, b);
}

ctc_status attn_args(const ctc_attention *c, AttnArgs &a) {
    if (!c) return fail(CTC_ERR_ARG, "NULL attention");
    if (c->dtype != CTC_F16 && c->dtype != CTC_BF16)
        return fail(CTC_ERR_ARG, "attention takes float16 or bfloat16");
    if (c->batch < 0 || c->queries < 0 || c->keys < 0 || c->q_heads < 1 || c->k_heads < 1)
        return fail(CTC_ERR_ARG, "bad attention sizes");
    if (c->q_heads % c->k_heads) return fail(CTC_ERR_ARG, "k_heads must divide q_heads");
    if (c->head < 8 || c->head % 8 || c->head > ATTN_MAX_D)
        return fail(CTC_ERR_ARG, "head sizes are multiples of 8 up to %d", ATTN_MAX_D);
    // (the kernels divide by it, and multiply it by log2 e)
    if (!(c->scale >= 0x1p-96f && c->scale <= 0x1p126f))
        return fail(CTC_ERR_ARG, "scale must be 2^-96 .. 2^126");
    const double rows = (double)c->queries * (c->q_heads / c->k_heads);
    const double pairs = (double)c->batch * c->k_heads;
    if (rows > (1 << 30) || c->keys > (1 << 30) || c->q_heads / c->k_heads > 65536 ||
        !grid_ok(pairs * (rows / 64 + (double)c->keys / 64 + 2) + 512))
        return fail(CTC_ERR_UNSUPPORTED, "attention too large");
    a = AttnArgs{};
    a.type = c->dtype;
    a.b = c->batch; a.tq = c->queries; a.tk = c->keys;
    a.hq = c->q_heads; a.hkv = c->k_heads; a.d = c->head;
    a.causal = c->causal != 0; a.scale = c->scale;
    a.qlen = c->q_lengths; a.klen = c->k_lengths;
    return CTC_OK;
}
ctc_status attn_heads(const AttnArgs &a, const ctc_heads *h, const char *name, bool queries,
                      bool out, const void *&data, int64_t (&strides)[3]) {
    const int64_t t = queries ? a.tq : a.tk, heads = queries ? a.hq : a.hkv;
    ctc_status s = heads_arg(h, name, a.b, t, heads, a.d, out, data, strides);
    if (s != CTC_OK) return s;
    if (!aligned(data, 16) || strides[0] % 8 || strides[1] % 8 || strides[2] % 8)
        return fail(CTC_ERR_ARG, "%s must be 16-byte aligned, its strides multiples of 8", name);
    // (a tile's addresses have 32 bits)
    const double group = queries ? a.hq / a.hkv : 1;
    if (64. * strides[1] + group * strides[2] >= (double)(1 << 29))
        return fail(CTC_ERR_UNSUPPORTED, "strides of %s too large", name);
    return CTC_OK;
}

struct Named {
    const char *name = "";
    Region r;
};
ctc_status meeting(const Named &x, const Named &y) {
    return fail(CTC_ERR_ARG, "%s overlaps %s", x.name, y.name);
}
Region attn_region(const AttnArgs &a, bool queries, const void *data, const int64_t (&strides)[3]) {
    return region(data, a.b, queries ? a.tq : a.tk, queries ? a.hq : a.hkv, strides, a.d, a.type);
}
Region attn_lse(const AttnArgs &a) {
    return dense(a.lse, (int64_t)a.b * a.hq * a.tq, CTC_F32);
}
// o may be q: a row is read and written by one wave, or written by the launch
// that joins ranges of keys.
ctc_status attn_apart(const AttnArgs &a) {
    const Named in[3] = {{"q", attn_region(a, true, a.q, a.qs)},
                         {"k", attn_region(a, false, a.k, a.ks)},
                         {"v", attn_region(a, false, a.v, a.vs)}};
    const Named out[2] = {{"o", attn_region(a, true, a.o, a.os)}, {"lse", attn_lse(a)}};
    if (meet(out[0].r, out[1].r)) return meeting(out[0], out[1]);
    for (int i = 0; i < 2; i++)
        for (int j = 0; j < 3; j++)
            if (!(i == 0 && j == 0 && out[i].r == in[j].r) && meet(out[i].r, in[j].r))
                return meeting(out[i], in[j]);
    return CTC_OK;
}
// dk and dv may be k and v: a workgroup reads the keys and values of the
// gradients that it writes and no others, so dq, which all keys go into, has to
// be there before (`keys_last`).
ctc_status attn_backward_apart(AttnArgs &a) {
    const Named in[6] = {{"dout", attn_region(a, true, a.dout, a.dos)},
                         {"q", attn_region(a, true, a.q, a.qs)},
                         {"o", attn_region(a, true, a.o, a.os)},
                         {"lse", attn_lse(a)},
                         {"k", attn_region(a, false, a.k, a.ks)},
                         {"v", attn_region(a, false, a.v, a.vs)}};
    const Named out[3] = {{"dq", attn_region(a, true, a.dq, a.dqs)},
                          {"dk", attn_region(a, false, a.dk, a.dks)},
                          {"dv", attn_region(a, false, a.dv, a.dvs)}};
    for (int i = 0; i < 3; i++) {
        for (int j = 0; j < i; j++)
            if (meet(out[i].r, out[j].r)) return meeting(out[i], out[j]);
        for (int j = 0; j < 6; j++) {
            if (!meet(out[i].r, in[j].r)) continue;
            if (i == 0 || j < 4 || !(out[i].r == in[j].r)) return meeting(out[i], in[j]);
            a.keys_last = 1;
        }
    }
    return CTC_OK;
}

// ------------------------------------------------------------ head norms

ctc_status head_args(const ctc_head_rotary *c, HeadArgs &a) {
    if (!c) return fail(CTC_ERR_ARG, "NULL head_rotary");
    if (!real_type(c->dtype) || !real_type(c->ytype) ||
        (c->dtype != CTC_F32 && c->ytype != c->dtype))
        return fail(CTC_ERR_ARG, "bad dtype");
    if (c->batch < 0 || c->tokens < 0 || c->q_heads < 1 || c->k_heads < 0)
        return fail(CTC_ERR_ARG, "bad head_norm_rotary sizes");
    if (c->head < 2 || c->head % 2 || c->head > 512)
        return fail(CTC_ERR_ARG, "head sizes are even, up to 512");
    if (!(c->eps >= 0.f) || std::isinf(c->eps)) return fail(CTC_ERR_ARG, "bad eps");
    if (c->axes < 0 || c->axes > 4) return fail(CTC_ERR_ARG, "up to 4 position axes");
    a = HeadArgs{};
    for (int i = 0; i < c->axes; i++) {
        if (c->pairs[i] < 0 || c->pairs[i] > c->head / 2)
            return fail(CTC_ERR_ARG, "bad pairs of an axis");
        a.axes[i] = c->pairs[i];
        a.turned += c->pairs[i];
    }
    if (a.turned > c->head / 2) return fail(CTC_ERR_ARG, "more pairs than a head has");
    a.type = c->dtype; a.ytype = c->ytype;
    a.b = c->batch; a.t = c->tokens; a.d = c->head;
    a.norm = c->norm != 0; a.eps = c->eps;
    a.interleaved = c->interleaved != 0; a.n_axes = c->axes; a.per_image = c->per_image != 0;
    a.positions = c->positions; a.frequencies = c->frequencies;
    a.side[0].heads = c->q_heads; a.side[0].weight = c->q_weight;
    a.side[1].heads = c->k_heads; a.side[1].weight = c->k_weight;
    if (!head_norm_ok(a) || (double)a.b * a.t >= (double)((int64_t)1 << 40) ||
        c->q_heads > (1 << 20) || c->k_heads > (1 << 20))
        return fail(CTC_ERR_UNSUPPORTED, "head_norm_rotary too large");
    return CTC_OK;
}
ctc_status head_positions(const HeadArgs &a) {
    if (a.turned && a.b && a.t && (!a.positions || !a.frequencies))
        return fail(CTC_ERR_ARG, "NULL positions or frequencies");
    return CTC_OK;
}
ctc_status head_side(const HeadArgs &a, int which, const ctc_heads *h, const char *name, bool out,
                     const void *&data, int64_t (&strides)[3]) {
    return heads_arg(h, name, a.b, a.t, a.side[which].heads, a.d, out, data, strides);
}

Region head_region(const HeadArgs &a, int which, const void *data, const int64_t (&strides)[3],
                   int type) {
    return region(data, a.b, a.t, a.side[which].heads, strides, a.d, type);
}
// A lane group reads a head before it writes it, so results may stand in the
// place of the head's own values; those of other heads are read at any time.
ctc_status head_apart(const HeadArgs &a, bool backward) {
    Named in[6], out[4];
    for (int i = 0; i < 2; i++) {
        const HeadSide &s = a.side[i];
        in[i] = {i ? "k" : "q", head_region(a, i, s.x, s.xs, a.type)};
        in[2 + i] = {i ? "k_weight" : "q_weight", dense(s.heads ? s.weight : nullptr, a.d, F32)};
        if (backward) {
            in[4 + i] = {i ? "dyk" : "dyq", head_region(a, i, s.dy, s.dys, a.ytype)};
            out[i] = {i ? "dk" : "dq", head_region(a, i, s.dx, s.dxs, a.type)};
            out[2 + i] = {i ? "dk_weight" : "dq_weight", dense(s.dweight, a.d, F32)};
        } else {
            out[i] = {i ? "yk" : "yq", head_region(a, i, s.y, s.ys, a.ytype)};
        }
    }
    for (int i = 0; i < (backward ? 4 : 2); i++) {
        for (int j = 0; j < i; j++)
            if (meet(out[i].r, out[j].r)) return meeting(out[i], out[j]);
        for (int j = 0; j < (backward ? 6 : 4); j++)
            if (meet(out[i].r, in[j].r) &&
                !(i < 2 && (j == i || j == 4 + i) && out[i].r == in[j].r))
                return meeting(out[i], in[j]);
    }
    return CTC_OK;
}

// --------------------------------------------------------------- clipping

ctc_status clip_args(int32_t n, const ctc_gradient *g) {
    if (n < 0 || (n && !g)) return fail(CTC_ERR_ARG, "bad gradients");
    if (n > (1 << 20)) return fail(CTC_ERR_UNSUPPORTED, "too many gradients");
    double chunks = 0;
    for (int32_t i = 0; i < n; i++) {
        if (!real_type(g[i].dtype)) return fail(CTC_ERR_ARG, "bad dtype of gradient %d", i);
        if (g[i].size < 0) return fail(CTC_ERR_ARG, "bad size of gradient %d", i);
        chunks += (double)g[i].size / (1 << 12) + 1;
        if (chunks >= 4294967295.) return fail(CTC_ERR_UNSUPPORTED, "gradients too large");
    }
    return CTC_OK;
}
// The launches' tables: f(table) for each CLIP_TENSORS tensors.
template <typename F> ctc_status clip_tables(int32_t n, const ctc_gradient *g, F f) {
    for (int32_t i = 0; i < n; i += CLIP_TENSORS) {
        ClipTable t;
        t.n = n - i < CLIP_TENSORS ? n - i : CLIP_TENSORS;
        t.first[0] = 0;
        for (int j = 0; j < t.n; j++) {
            t.x[j] = g[i + j].x;
            t.y[j] = g[i + j].y;
            t.size[j] = g[i + j].size;
            t.type[j] = (uint8_t)g[i + j].dtype;
            t.first[j + 1] = t.first[j] + (uint32_t)clip_chunks_of(g[i + j].size);
        }
        ctc_status s = f(t);
        if (s != CTC_OK) return s;
    }
    return CTC_OK;
}
// No output (the norm among them) overlaps another one, or another tensor's
// values.
bool clip_disjoint(int32_t n, const ctc_gradient *g, const float *norm) {
    struct Span { uintptr_t from, to; int32_t i; };
    std::vector<Span> out, in;
    out.reserve(n + 1);
    in.reserve(n);
    if (norm) out.push_back({(uintptr_t)norm, (uintptr_t)(norm + 1), -1});
    for (int32_t i = 0; i < n; i++) {
        const size_t bytes = (size_t)g[i].size * type_bytes(g[i].dtype);
        if (!bytes) continue;
        out.push_back({(uintptr_t)g[i].y, (uintptr_t)g[i].y + bytes, i});
        if (g[i].y != g[i].x) in.push_back({(uintptr_t)g[i].x, (uintptr_t)g[i].x + bytes, i});
    }
    auto order = [](const Span &a, const Span &b) { return a.from < b.from; };
    std::sort(out.begin(), out.end(), order);
    for (size_t i = 1; i < out.size(); i++)
        if (out[i].from < out[i - 1].to) return false;
    for (const Span &s : in) {
        // the first output that ends behind s begins
        auto it = std::upper_bound(out.begin(), out.end(), s.from,
                                   [](uintptr_t v, const Span &o) { return v < o.to; });
        if (it != out.end() && it->from < s.to) return false;
    }
    return true;
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

ctc_status ctc_attention_workspace_bytes(const ctc_attention *c, int32_t backward, size_t *bytes) {
    if (!bytes) return fail(CTC_ERR_ARG, "NULL bytes");
    AttnArgs a;
    ctc_status s = attn_args(c, a);
    if (s != CTC_OK) return s;
    *bytes = a.b && (backward || a.tq) ? attention_workspace(a, backward != 0) : 0;
    return CTC_OK;
}

ctc_status ctc_attention_forward(const ctc_attention *c, const ctc_heads *q, const ctc_heads *k,
                                 const ctc_heads *v, const ctc_heads *o, float *lse,
                                 void *workspace, size_t ws_bytes, void *stream) {
    AttnArgs a;
    ctc_status s = attn_args(c, a);
    if (s != CTC_OK) return s;
    if (a.b == 0 || a.tq == 0) return CTC_OK;
    const void *out = nullptr;
    if ((s = attn_heads(a, q, "q", true, false, a.q, a.qs)) != CTC_OK ||
        (s = attn_heads(a, k, "k", false, false, a.k, a.ks)) != CTC_OK ||
        (s = attn_heads(a, v, "v", false, false, a.v, a.vs)) != CTC_OK ||
        (s = attn_heads(a, o, "o", true, true, out, a.os)) != CTC_OK)
        return s;
    if (!lse) return fail(CTC_ERR_ARG, "NULL lse");
    a.o = (void *)out; a.lse = lse; a.ws = (float *)workspace;
    s = need_workspace(attention_workspace(a, false), workspace, ws_bytes);
    if (s != CTC_OK || (s = attn_apart(a)) != CTC_OK) return s;
    return done(launch_attention(a, S(stream)));
}

ctc_status ctc_attention_backward(const ctc_attention *c, const ctc_heads *dout,
                                  const ctc_heads *q, const ctc_heads *k, const ctc_heads *v,
                                  const ctc_heads *o, const float *lse, const ctc_heads *dq,
                                  const ctc_heads *dk, const ctc_heads *dv, void *workspace,
                                  size_t ws_bytes, void *stream) {
    AttnArgs a;
    ctc_status s = attn_args(c, a);
    if (s != CTC_OK) return s;
    if (a.b == 0 || (a.tq == 0 && a.tk == 0)) return CTC_OK;
    const void *op = nullptr, *dqp = nullptr, *dkp = nullptr, *dvp = nullptr;
    if ((s = attn_heads(a, dout, "dout", true, false, a.dout, a.dos)) != CTC_OK ||
        (s = attn_heads(a, q, "q", true, false, a.q, a.qs)) != CTC_OK ||
        (s = attn_heads(a, k, "k", false, false, a.k, a.ks)) != CTC_OK ||
        (s = attn_heads(a, v, "v", false, false, a.v, a.vs)) != CTC_OK ||
        (s = attn_heads(a, o, "o", true, false, op, a.os)) != CTC_OK ||
        (s = attn_heads(a, dq, "dq", true, true, dqp, a.dqs)) != CTC_OK ||
        (s = attn_heads(a, dk, "dk", false, true, dkp, a.dks)) != CTC_OK ||
        (s = attn_heads(a, dv, "dv", false, true, dvp, a.dvs)) != CTC_OK)
        return s;
    if (a.tq && !lse) return fail(CTC_ERR_ARG, "NULL lse");
    a.o = (void *)op; a.lse = (float *)lse; a.ws = (float *)workspace;
    a.dq = (void *)dqp; a.dk = (void *)dkp; a.dv = (void *)dvp;
    s = need_workspace(attention_workspace(a, true), workspace, ws_bytes);
    if (s != CTC_OK || (s = attn_backward_apart(a)) != CTC_OK) return s;
    return done(launch_attention_backward(a, S(stream)));
}

ctc_status ctc_head_norm_rotary_workspace_bytes(const ctc_head_rotary *c, size_t *bytes) {
    if (!bytes) return fail(CTC_ERR_ARG, "NULL bytes");
    HeadArgs a;
    ctc_status s = head_args(c, a);
    if (s != CTC_OK) return s;
    *bytes = head_norm_workspace(a);
    return CTC_OK;
}

ctc_status ctc_head_norm_rotary_forward(const ctc_head_rotary *c, const ctc_heads *q,
                                        const ctc_heads *k, const ctc_heads *yq,
                                        const ctc_heads *yk, void *stream) {
    HeadArgs a;
    ctc_status s = head_args(c, a);
    if (s != CTC_OK || (s = head_positions(a)) != CTC_OK) return s;
    const ctc_heads *x[2] = {q, k}, *y[2] = {yq, yk};
    for (int i = 0; i < 2; i++) {
        HeadSide &h = a.side[i];
        const void *out = nullptr;
        if ((s = head_side(a, i, x[i], i ? "k" : "q", false, h.x, h.xs)) != CTC_OK ||
            (s = head_side(a, i, y[i], i ? "yk" : "yq", true, out, h.ys)) != CTC_OK)
            return s;
        h.y = (void *)out;
    }
    if ((s = head_apart(a, false)) != CTC_OK) return s;
    return done(launch_head_norm(a, false, S(stream)));
}

ctc_status ctc_head_norm_rotary_backward(const ctc_head_rotary *c, const ctc_heads *dyq,
                                         const ctc_heads *dyk, const ctc_heads *q,
                                         const ctc_heads *k, const ctc_heads *dq,
                                         const ctc_heads *dk, float *dq_weight, float *dk_weight,
                                         void *workspace, size_t ws_bytes, void *stream) {
    HeadArgs a;
    ctc_status s = head_args(c, a);
    if (s != CTC_OK || (s = head_positions(a)) != CTC_OK) return s;
    const ctc_heads *x[2] = {q, k}, *dy[2] = {dyq, dyk}, *dx[2] = {dq, dk};
    for (int i = 0; i < 2; i++) {
        HeadSide &h = a.side[i];
        const void *out = nullptr;
        if ((s = head_side(a, i, x[i], i ? "k" : "q", false, h.x, h.xs)) != CTC_OK ||
            (s = head_side(a, i, dy[i], i ? "dyk" : "dyq", false, h.dy, h.dys)) != CTC_OK ||
            (s = head_side(a, i, dx[i], i ? "dk" : "dq", true, out, h.dxs)) != CTC_OK)
            return s;
        h.dx = (void *)out;
    }
    a.side[0].dweight = dq_weight;
    a.side[1].dweight = a.side[1].heads ? dk_weight : nullptr;
    a.ws = (float *)workspace;
    s = need_workspace(head_norm_workspace(a), workspace, ws_bytes);
    if (s != CTC_OK || (s = head_apart(a, true)) != CTC_OK) return s;
    return done(launch_head_norm(a, true, S(stream)));
}

ctc_status ctc_clip_gradients_workspace_bytes(int32_t n, const ctc_gradient *g, size_t *bytes) {
    if (!bytes) return fail(CTC_ERR_ARG, "NULL bytes");
    ctc_status s = clip_args(n, g);
    if (s != CTC_OK) return s;
    size_t parts = 0;
    s = clip_tables(n, g, [&](const ClipTable &t) {
        parts += clip_parts(t);
        return CTC_OK;
    });
    *bytes = parts * sizeof(double);
    return s;
}

ctc_status ctc_clip_gradients(int32_t n, const ctc_gradient *g, float max_norm, float *norm,
                              void *workspace, size_t ws_bytes, void *stream) {
    return ctc_clip_gradients_to(n, g, max_norm, norm, workspace, ws_bytes, stream);
}

ctc_status ctc_clip_gradients_to(int32_t n, const ctc_gradient *g, double max_norm, float *norm,
                                 void *workspace, size_t ws_bytes, void *stream) {
    size_t need = 0;
    ctc_status s = ctc_clip_gradients_workspace_bytes(n, g, &need);
    if (s != CTC_OK) return s;
    if (!(max_norm >= 0)) return fail(CTC_ERR_ARG, "max_norm must be >= 0");
    for (int32_t i = 0; i < n; i++)
        if (g[i].size && (!g[i].x || !g[i].y)) return fail(CTC_ERR_ARG, "NULL gradient %d", i);
    try {
        if (!clip_disjoint(n, g, norm)) return fail(CTC_ERR_ARG, "outputs overlap other gradients");
    } catch (const std::exception &e) {
        return fail(CTC_ERR_DEVICE, "%s", e.what());
    }
    s = need_workspace(need, workspace, ws_bytes);
    if (s != CTC_OK) return s;
    double *part = (double *)workspace;
    int parts = 0;
    s = clip_tables(n, g, [&](const ClipTable &t) {
        const ctc_status r = done(launch_clip_squares(t, part + parts, S(stream)));
        parts += clip_parts(t);
        return r;
    });
    if (s != CTC_OK) return s;
    if (!n) {
        if (!norm) return CTC_OK;
        ClipTable t;
        t.n = 0;
        t.first[0] = 0;
        return done(launch_clip_scale(t, part, 0, max_norm, norm, S(stream)));
    }
    return clip_tables(n, g, [&](const ClipTable &t) {
        return done(launch_clip_scale(t, part, parts, max_norm, norm, S(stream)));
    });
}

}  // extern "C"
