"""Attention and its backward pass against the formulas in 64 bits.

Tolerances follow from the arithmetic.  With u half a step of the type (2^-11
or 2^-8): a score is a sum of d products in fp32, off by d 2^-24 of the
products' magnitudes; with its rounding in the exponent that is the relative
error of a probability (E below).  Probabilities are rounded to the type before
they meet v (u each), o once more.  For fp16 a probability is kept as p 2^8 of
the row's largest or more: its subnormals cost 2^-33 of it.  The backward pass
rounds p and ds (u each, in fp16 at least 2^-25 of 2^-e for the exponent e that
the sequence's gradients allow), and takes delta from the rounded o.  Below
2^-126, the least normal number of fp32 and of bf16, probabilities and results
may be zeros: exp(-88) and less, which scores of hundreds reach.
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f16": torch.float16, "bf16": torch.bfloat16}
U = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}
LEAST = 2.0 ** -126
INF = math.inf


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import ops
    return ops


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _within(got, want, bound, what):
    got, want = got.double(), want.double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(got[~fine].nan_to_num(0), want[~fine].nan_to_num(0)), what
    off = (got - want).abs()
    over = fine & ~(off <= bound)
    if bool(over.any()):
        i = int((off / bound.clamp(min=1e-300)).masked_fill(~over, 0).argmax())
        raise AssertionError("%s: %d of %d off, worst at %d: %.9g for %.9g, bound %.3g" % (
            what, int(over.sum()), over.numel(), i, got.flatten()[i],
            want.flatten()[i], bound.flatten()[i]))


def _lengths(n, b, t, values):
    if values is None:
        return [t] * b
    return [min(max(int(v), 0), t) for v in values]


class Case:
    """Inputs of a call, and the formulas in 64 bits with their bounds."""

    def __init__(self, dtype, b, tq, tk, hq, hkv, d, causal=False,
                 q_lengths=None, k_lengths=None, scale=None, seed=1, size=1.0,
                 dsize=1.0):
        g = _gen(seed)
        self.dtype, self.u, self.causal = dtype, U[dtype], causal
        self.b, self.tq, self.tk, self.hq, self.hkv, self.d = b, tq, tk, hq, hkv, d
        self.scale = d ** -0.5 if scale is None else scale
        # parts of projections: strided in tokens and heads
        qkv = (_randn(g, b, max(tq, tk), hq + 2 * hkv, d) * size).to(DT[dtype])
        self.q = qkv[:, :tq, :hq]
        self.k = qkv[:, :tk, hq:hq + hkv]
        self.v = qkv[:, :tk, hq + hkv:]
        self.do = (_randn(g, b, tq, hq, d) * dsize).to(DT[dtype])

        def dev(v):
            return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")
        self.nq, self.nk = _lengths(b, b, tq, q_lengths), _lengths(b, b, tk, k_lengths)
        self.kw = dict(causal=causal, q_lengths=dev(q_lengths),
                       k_lengths=dev(k_lengths), scale=scale)

    def reference(self):
        f8 = dict(dtype=torch.float64, device="cuda")
        b, tq, tk, hq, hkv, d = self.b, self.tq, self.tk, self.hq, self.hkv, self.d
        u = self.u
        out = {n: torch.zeros((b, tq, hq, d), **f8) for n in ("o", "dq")}
        out.update({n: torch.zeros((b, tk, hkv, d), **f8) for n in ("dk", "dv")})
        out["lse"] = torch.full((b, hq, tq), -INF, **f8)
        tol = {n: torch.zeros_like(t) for n, t in out.items()}
        for i in range(b):
            nq, nk = self.nq[i], self.nk[i]
            if not nq or not nk:
                continue
            hide = torch.zeros((nq, nk), dtype=torch.bool, device="cuda")
            if self.causal:
                hide = (torch.arange(nk, device="cuda")[None] >
                        torch.arange(nq, device="cuda")[:, None] + nk - nq)
            gone = hide.all(1, keepdim=True)
            for h in range(hq):
                kh = h // (hq // hkv)
                q, k = self.q[i, :nq, h].double(), self.k[i, :nk, kh].double()
                v, do = self.v[i, :nk, kh].double(), self.do[i, :nq, h].double()
                do = torch.where(gone, 0.0, do)
                # (what a row does not see reaches it in no way)
                s = torch.where(hide, -INF, (q @ k.t()) * self.scale)
                mag = torch.where(hide, 0.0, (q.abs() @ k.abs().t()) * self.scale)
                lse = torch.logsumexp(s, 1, keepdim=True)
                p = torch.where(hide | gone, 0.0, torch.exp(s - lse))
                o = p @ v
                # relative error of a probability
                safe = torch.where(gone, 0.0, lse.abs())
                e = (mag * (d + 4) * 2.0 ** -24 + torch.where(hide, 0.0, s.abs()) * 2.0 ** -22
                     + 2.0 ** -21).amax(1, keepdim=True) + safe * 2.0 ** -22
                e_o = 2 * e + nk * 2.0 ** -24
                small = 2.0 ** -33 if self.dtype == "f16" else LEAST
                to = (p @ v.abs()) * (e_o + u) + u * o.abs() + small * (
                    p.amax(1, keepdim=True) * v.abs().sum(0)[None]) + (
                        2.0 ** -25 if self.dtype == "f16" else LEAST)
                out["o"][i, :nq, h], tol["o"][i, :nq, h] = o, to
                out["lse"][i, h, :nq], tol["lse"][i, h, :nq] = lse[:, 0], \
                    (e + nk * 2.0 ** -24)[:, 0]
                # backward
                ex = 0.0
                if self.dtype == "f16":
                    nv = self.v[i, :nk, kh].double().norm(dim=1).max()
                    grp = range(kh * (hq // hkv), (kh + 1) * (hq // hkv))
                    nd = max(float(torch.where(gone[:, 0], 0.0, self.do[i, :nq, x].double()
                                               .norm(dim=1)).max()) for x in grp)
                    ex = min(15.0, max(-20.0, 13.0 - math.ceil(
                        1 + math.log2(max(1e-300, nd * float(nv))))))
                floor = 2.0 ** (-25 - ex) if self.dtype == "f16" else LEAST
                dp, dpa = do @ v.t(), do.abs() @ v.abs().t()
                delta = (do * o).sum(1, keepdim=True)
                delta_off = (do.abs() * to).sum(1, keepdim=True) + (
                    do.abs() * o.abs()).sum(1, keepdim=True) * d * 2.0 ** -23
                ds = p * (dp - delta)
                # (two relative errors of p: lse as it was rounded, and its own)
                ds_off = p * ((2 * e + u) * (dp - delta).abs() + dpa * d * 2.0 ** -23
                              + delta_off) * (1 + u) + torch.where(hide, 0.0, floor)
                p_off = p * (2 * e + u) + torch.where(hide, 0.0, floor)
                sums = 2.0 ** -24
                out["dv"][i, :nk, kh] += p.t() @ do
                tol["dv"][i, :nk, kh] += (p_off + p * nq * sums).t() @ do.abs()
                out["dk"][i, :nk, kh] += self.scale * (ds.t() @ q)
                tol["dk"][i, :nk, kh] += self.scale * (
                    (ds_off + ds.abs() * nq * sums).t() @ q.abs())
                out["dq"][i, :nq, h] = self.scale * (ds @ k)
                tol["dq"][i, :nq, h] = self.scale * ((ds_off + ds.abs() * nk * sums) @ k.abs())
        for n in ("dq", "dk", "dv"):
            tol[n] += u * out[n].abs() + (2.0 ** -25 if self.dtype == "f16" else LEAST)
        return out, tol

    def check(self, ops, backward=True):
        want, tol = self.reference()
        o, lse = ops.attention(self.q, self.k, self.v, **self.kw)
        _within(o, want["o"], tol["o"], "o")
        _within(lse, want["lse"], tol["lse"], "lse")
        if backward:
            dq, dk, dv = ops.attention_backward(self.do, self.q, self.k, self.v, o, lse, **self.kw)
            _within(dv, want["dv"], tol["dv"], "dv")
            _within(dq, want["dq"], tol["dq"], "dq")
            _within(dk, want["dk"], tol["dk"], "dk")


# b, tq, tk, hq, hkv, head size: one of each, tiles and their edges, heads that
# share keys, sizes that are no whole steps
SHAPES = [(1, 1, 1, 1, 1, 8), (2, 49, 49, 8, 8, 64), (1, 64, 64, 1, 1, 128),
          (1, 65, 63, 2, 1, 128), (3, 33, 130, 3, 3, 40), (2, 129, 257, 4, 2, 72),
          (1, 196, 196, 12, 4, 80), (2, 1, 300, 32, 8, 128), (1, 3, 1000, 4, 1, 96),
          (1, 500, 2, 5, 5, 32), (1, 130, 70, 8, 1, 16), (8, 5, 7, 2, 2, 64),
          (1, 260, 390, 7, 1, 104)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_attention(ops, shape, causal, dtype):
    Case(dtype, *shape, causal=causal).check(ops)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_lengths(ops, causal, dtype):
    """None, one, all, and more or fewer than there are (clamped); rows that
    see nothing."""
    Case(dtype, 6, 70, 140, 4, 2, 64, causal=causal,
         q_lengths=[70, 1, 0, 33, 64, 1000], k_lengths=[140, 0, 17, 1, 65, -3]).check(ops)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("d", [16, 64, 80, 128])
def test_small_lengths(ops, d, causal, dtype):
    """Sequences that one workgroup takes whole, rows of shared heads among
    them."""
    Case(dtype, 6, 20, 50, 6, 2, d, causal=causal, q_lengths=[20, 1, 0, 13, 20, 99],
         k_lengths=[50, 0, 17, 1, 33, -3]).check(ops)
    Case(dtype, 3, 64, 64, 2, 2, d, causal=causal, q_lengths=[64, 63, 33],
         k_lengths=[64, 31, 33]).check(ops)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_long_keys(ops, dtype):
    """Few rows over many keys (ranges of keys joined), and their gradients."""
    Case(dtype, 2, 1, 12544, 8, 2, 128, k_lengths=[12544, 5000]).check(ops)
    Case(dtype, 1, 2, 9001, 3, 3, 64, causal=True).check(ops)
    Case(dtype, 1, 200, 7001, 1, 1, 40).check(ops)
    Case(dtype, 2, 150, 4000, 2, 1, 72, causal=True, q_lengths=[150, 100],
         k_lengths=[2100, 4000]).check(ops)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_long_rows(ops, dtype):
    Case(dtype, 1, 3000, 40, 4, 1, 64).check(ops)
    Case(dtype, 1, 1025, 1025, 4, 2, 128, causal=True).check(ops)


# ------------------------------------------------- NaN and infinite values

@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("t,d", [(40, 64), (200, 64), (200, 128), (30, 128)])
def test_what_stands_behind_the_lengths(ops, t, d, dtype, causal):
    """NaN and infinities there reach nothing, forward or backward."""
    c = Case(dtype, 3, t, t, 4, 2, d, causal=causal, q_lengths=[t, t // 2, 0],
             k_lengths=[t - 1, 7, 5])
    o, lse = ops.attention(c.q, c.k, c.v, **c.kw)
    want = (o, lse) + ops.attention_backward(c.do, c.q, c.k, c.v, o, lse, **c.kw)
    bad = {}
    for n in ("q", "k", "v", "do"):
        x = getattr(c, n).clone()
        for i in range(3):
            x[i, (c.nq if n in ("q", "do") else c.nk)[i]:] = math.nan if n != "v" else INF
        bad[n] = x
    o2, lse2 = ops.attention(bad["q"], bad["k"], bad["v"], **c.kw)
    # (o behind the queries' lengths is zeros as written; the backward pass does
    # not read it)
    o3 = o2.clone()
    for i in range(3):
        o3[i, c.nq[i]:] = math.nan
    got = (o2, lse2) + ops.attention_backward(bad["do"], bad["q"], bad["k"], bad["v"], o3, lse2,
                                              **c.kw)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def _causal_case(ops, t, d, plant):
    """(baseline, results with a value planted) of a causal case in bf16."""
    c = Case("bf16", 2, t, t, 4, 2, d, causal=True)
    x = {n: getattr(c, n).clone() for n in ("q", "k", "v", "do")}

    def run():
        o, lse = ops.attention(x["q"], x["k"], x["v"], causal=True)
        g = ops.attention_backward(x["do"], x["q"], x["k"], x["v"], o, lse, causal=True)
        return dict(zip(("o", "lse", "dq", "dk", "dv"), (o, lse.transpose(1, 2)) + g))
    want = run()
    plant(x)
    return want, run()



@pytest.mark.parametrize("value", [math.nan, INF, -INF])
@pytest.mark.parametrize("t,d", [(50, 64), (50, 128), (64, 32), (200, 64), (200, 128), (333, 96)])
def test_values_that_causal_queries_do_not_see(ops, t, d, value):
    """One NaN or infinity at token j: what does not see it stays as it was,
    bit for bit, and what does shows it."""
    for j in (0, 1, t // 2, t - 2, t - 1):
        before, after = slice(0, j), slice(j, t)
        e = 5 % d

        def put(n):
            def f(x):
                x[n][0, j, 0, e] = value
            return f
        # heads 0 and 1 share key head 0 of sequence 0; the rest sees nothing
        def rest(got, want):
            for n in got:
                assert torch.equal(got[n][1], want[n][1]), n
                heads = 1 if n in ("dk", "dv") else 2
                assert torch.equal(got[n][0, :, heads:], want[n][0, :, heads:]), n
        want, got = _causal_case(ops, t, d, put("v"))
        rest(got, want)
        for n in ("o", "lse", "dq", "dv"):
            assert torch.equal(got[n][0, before], want[n][0, before]), n
        assert torch.equal(got["lse"], want["lse"]) and torch.equal(got["dv"], want["dv"])
        assert not bool(torch.isfinite(got["o"][0, after, :2, e]).any())
        keep = [i for i in range(d) if i != e]
        assert torch.equal(got["o"][0, after, :2][..., keep], want["o"][0, after, :2][..., keep])
        assert not bool(torch.isfinite(got["dq"][0, after, :2].float()).any())
        if math.isnan(value):
            want, got = _causal_case(ops, t, d, put("k"))
            rest(got, want)
            for n in ("o", "lse", "dq"):
                assert torch.equal(got[n][0, before], want[n][0, before]), n
                assert bool(torch.isnan(got[n][0, after, :2]).all()), n
            want, got = _causal_case(ops, t, d, put("q"))
            rest(got, want)
            others = [i for i in range(t) if i != j]
            for n in ("o", "lse", "dq"):
                assert torch.equal(got[n][0, others], want[n][0, others]), n
                assert bool(torch.isnan(got[n][0, j, 0]).all()), n
            for n in ("dk", "dv"):
                assert torch.equal(got[n][0, j + 1:], want[n][0, j + 1:]), n
                assert bool(torch.isnan(got[n][0, :j + 1, 0]).all()), n
        want, got = _causal_case(ops, t, d, put("do"))
        rest(got, want)
        others = [i for i in range(t) if i != j]
        assert torch.equal(got["dq"][0, others], want["dq"][0, others])
        assert not bool(torch.isfinite(got["dq"][0, j, 0].float()).any())
        for n in ("dk", "dv"):
            assert torch.equal(got[n][0, j + 1:], want[n][0, j + 1:]), n
        assert not bool(torch.isfinite(got["dk"][0, :j + 1, 0].float()).any())
        assert not bool(torch.isfinite(got["dv"][0, :j + 1, 0, e].float()).any())
        assert torch.equal(got["dv"][0, :j + 1, 0][..., keep], want["dv"][0, :j + 1, 0][..., keep])
