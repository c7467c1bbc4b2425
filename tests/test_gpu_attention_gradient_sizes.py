"""Attention's gradients in fp16 where gradients and values are large, small, or
large in one place, against the formulas in 64 bits.

Tolerances as in test_gpu_attention.py (u = 2^-11 is half a step, E the relative
error of a probability), but for what fp16's range takes:
  * p for dv is kept at 2^15 p, which is at most 2^15: half a subnormal step,
    2^-25, is 2^-40 of it, whatever the gradients' sizes are.
  * ds is kept at 2^e ds, with e such that 2 |do| |v| 2^e is 2^13 or more (and
    2^60 at most): 2^-25-e.  |v| is the largest of the sequence and key head.
    |do| is the row's own for dq, and the largest of the rows for dk, whose sums
    go over them.
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import _gen, _randn, _within  # noqa: E402

U = 2.0 ** -11


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import ops
    return ops


def _exponent(do, v):
    """e of 64-bit sizes, one less for the rounding of its logarithms."""
    return (13 - torch.ceil(1 + torch.log2((do * v).clamp(min=1e-300)))).clamp(max=60.0)


def _reference(q, k, v, do, scale, causal):
    """dq, dk, dv and their bounds, of one sequence [tokens, heads, size]."""
    q, k, v, do = (t.double() for t in (q, k, v, do))
    (nq, hq, d), (nk, hk) = q.shape, k.shape[:2]
    want = {"dq": torch.zeros_like(q), "dk": torch.zeros_like(k), "dv": torch.zeros_like(v)}
    tol = {n: torch.zeros_like(t) for n, t in want.items()}
    hide = torch.zeros((nq, nk), dtype=torch.bool, device="cuda")
    if causal:
        hide = (torch.arange(nk, device="cuda")[None] >
                torch.arange(nq, device="cuda")[:, None] + nk - nq)
    gone = hide.all(1, keepdim=True)
    for h in range(hq):
        kh = h // (hq // hk)
        group = slice(kh * (hq // hk), (kh + 1) * (hq // hk))
        qh, kk, vv = q[:, h], k[:, kh], v[:, kh]
        g = torch.where(gone, 0.0, do[:, h])
        s = torch.where(hide, -math.inf, (qh @ kk.t().contiguous()) * scale)
        mag = torch.where(hide, 0.0, (qh.abs() @ kk.abs().t().contiguous()) * scale)
        lse = torch.logsumexp(s, 1, keepdim=True)
        p = torch.where(hide | gone, 0.0, torch.exp(s - lse))
        o = p @ vv
        e = (mag * (d + 4) * 2.0 ** -24 + torch.where(hide, 0.0, s.abs()) * 2.0 ** -22
             + 2.0 ** -21).amax(1, keepdim=True) + torch.where(gone, 0.0, lse.abs()) * 2.0 ** -22
        to = (p @ vv.abs()) * (2 * e + nk * 2.0 ** -24 + U) + U * o.abs() + 2.0 ** -33 * (
            p.amax(1, keepdim=True) * vv.abs().sum(0)[None]) + 2.0 ** -25
        most = vv.norm(dim=1).max()
        rows = torch.where(gone, 0.0, g.norm(dim=1, keepdim=True))
        all_rows = torch.where(gone[:, 0, None], 0.0, do[:, group].norm(dim=2)).max()
        seen = (~hide).double()
        floor_q = 2.0 ** (-25 - _exponent(rows, most)) * seen
        floor_k = 2.0 ** (-25 - _exponent(all_rows, most)) * seen
        dp, dpa = g @ vv.t().contiguous(), g.abs() @ vv.abs().t().contiguous()
        delta = (g * o).sum(1, keepdim=True)
        delta_off = (g.abs() * to).sum(1, keepdim=True) + (
            g.abs() * o.abs()).sum(1, keepdim=True) * d * 2.0 ** -23
        ds = p * (dp - delta)
        ds_off = p * ((2 * e + U) * (dp - delta).abs() + dpa * d * 2.0 ** -23
                      + delta_off) * (1 + U)
        p_off = p * (2 * e + U) + 2.0 ** -40 * seen
        sums = 2.0 ** -24
        want["dv"][:, kh] += p.t() @ g
        tol["dv"][:, kh] += (p_off + p * nq * sums).t() @ g.abs()
        want["dk"][:, kh] += scale * (ds.t() @ qh)
        tol["dk"][:, kh] += scale * ((ds_off + floor_k + ds.abs() * nq * sums).t() @ qh.abs())
        want["dq"][:, h] = scale * (ds @ kk)
        tol["dq"][:, h] = scale * ((ds_off + floor_q + ds.abs() * nk * sums) @ kk.abs())
    for n in want:
        tol[n] += U * want[n].abs() + 2.0 ** -25
    return want, tol


def _check(ops, q, k, v, do, causal=False):
    scale = q.shape[-1] ** -0.5
    q, k, v, do = (t.half() for t in (q, k, v, do))
    o, lse = ops.attention(q[None], k[None], v[None], causal=causal)
    got = ops.attention_backward(do[None], q[None], k[None], v[None], o, lse, causal=causal)
    want, tol = _reference(q, k, v, do, scale, causal)
    for n, t in zip(("dq", "dk", "dv"), got):
        # (65520 and more is infinite in fp16, by its sign)
        t, w, size = t[0], want[n], want[n].abs()
        inf = torch.isinf(t)
        assert bool((inf | (size - tol[n] < 65520)).all()), n
        assert bool((~inf | ((size + tol[n] >= 65520) & (t.sign() == w.sign()))).all()), n
        _within(t[~inf], w[~inf], tol[n][~inf], n)
    return got, want


def _inputs(nq, nk, hq, hk, d, seed=1):
    g = _gen(seed)
    return (_randn(g, nq, hq, d), _randn(g, nk, hk, d), _randn(g, nk, hk, d), _randn(g, nq, hq, d))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape,dsize,vsize", [
    ((200, 3136, 1, 1, 128), 4000.0, 4.0), ((64, 12544, 1, 1, 64), 4000.0, 8.0),
    ((1, 12544, 4, 1, 128), 2000.0, 2.0), ((300, 700, 4, 2, 64), 4000.0, 4.0),
    ((50, 60, 4, 2, 64), 2000.0, 8.0), ((64, 64, 1, 1, 128), 1000.0, 8.0)], ids=str)
def test_large(ops, shape, dsize, vsize, causal):
    q, k, v, do = _inputs(*shape)
    _check(ops, q, k / 8, v * vsize, do * dsize, causal)


@pytest.mark.parametrize("nk", [64, 3136])
def test_equal_scores(ops, nk):
    """Every probability is 1 / keys."""
    q, k, v, do = _inputs(60, nk, 2, 1, 64)
    _check(ops, q * 0, k / 16, v * 8, do * 4000)


@pytest.mark.parametrize("shape", [(64, 64, 2, 2, 64), (64, 64, 1, 1, 128), (200, 300, 2, 2, 96),
                                   (100, 3000, 1, 1, 32)], ids=str)
def test_largest(ops, shape):
    """Gradients and values next to the type's largest."""
    q, k, v, do = _inputs(*shape)
    _check(ops, q / 256, k / 32768, v.clamp(-2, 2) * 16000, do.clamp(-2, 2) * 30000)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(60, 64, 4, 2, 64), (64, 64, 1, 1, 128), (400, 600, 2, 1, 64),
                                   (400, 600, 2, 1, 128)], ids=str)
def test_one_large_row(ops, shape, causal):
    """A row whose gradient is 2^23 times the others': these keep their dq."""
    q, k, v, do = _inputs(*shape)
    large = do[17].clamp(-1, 1) * 2.0 ** 15
    do = do / 256
    do[17] = large
    got, want = _check(ops, q, k, v, do, causal)
    keep = [i for i in range(shape[0]) if i != 17]
    a, b = got[0][0].double()[keep], want["dq"][keep]
    # (half a step of fp16 of p, of ds and of o each, and of dq, whose own least
    # step is 2^-24)
    assert float((a - b).norm()) <= 4 * U * float(b.norm()) + 2.0 ** -25 * math.sqrt(b.numel())


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(60, 64, 4, 2, 64), (400, 600, 2, 1, 128)], ids=str)
def test_one_large_value(ops, shape, causal):
    q, k, v, do = _inputs(*shape)
    v[5] = v[5].clamp(-2, 2) * 30000
    _check(ops, q, k / 64, v, do, causal)


@pytest.mark.parametrize("shape", [(60, 64, 4, 2, 64), (400, 600, 2, 1, 128)], ids=str)
def test_small_gradients_of_large_keys(ops, shape):
    """ds far below fp16's least step, which keys and queries make large."""
    q, k, v, do = _inputs(*shape)
    k = torch.cat([k[..., :1] * 0 + 4000, k[..., 1:]], -1)     # (adds the same to a row's scores)
    q = torch.cat([q[..., :1] * 0 + 2.0 ** -8, q[..., 1:] / 8], -1)
    _check(ops, q, k, v / 64, do * 2.0 ** -12)
