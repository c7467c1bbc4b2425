"""Norms of heads whose squares leave fp32: values of any size the type holds.

Tolerances as in test_gpu_head_norm.py: a mean of d squares is off by d 2^-24 of
it, its root and reciprocal by two roundings, a result by half a step of its type
(which below the type's normal numbers is half its least step)."""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_head_norm import DT, U, _within  # noqa: E402

LEAST = {"f32": 2.0 ** -150, "bf16": 2.0 ** -134, "f16": 2.0 ** -25}


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import ops
    return ops


def _case(dtype, d, sizes, seed):
    """Heads of the given sizes in turn, side by side in a wave."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn((2, 9, len(sizes), d), device="cuda", generator=g).clamp(-3, 3)
    x = (x.double() * torch.tensor(sizes, dtype=torch.float64, device="cuda")[:, None]).to(DT[dtype])
    w = 1 + 0.3 * torch.randn(d, device="cuda", generator=g)
    dy = torch.randn(x.shape, device="cuda", generator=g).to(DT[dtype])
    return x, w, dy


@pytest.mark.parametrize("d", [2, 6, 64, 80, 128, 512])
@pytest.mark.parametrize("dtype,sizes,eps", [
    ("f32", (1.0, 1e25, 1e38, 1e19, 1e10, 3.0), 1e-6),
    ("bf16", (1.0, 1e25, 1e38, 1e19, 1e10), 1e-6),
    ("f32", (1.0, 1e-25, 1e-36, 1e-18, 1e38, 1e-12), 0.0),
    ("bf16", (1.0, 1e-25, 1e-36, 1e-18, 1e38), 0.0),
    ("f32", (1.0, 1e-25, 1e-42, 1e-5), 1e-6), ("f16", (1.0, 1e-7, 2e4), 0.0),
    ("f32", (1e-20, 1e-16, 1e-15, 1e-14), 1e-33)], ids=str)
def test_sizes(ops, dtype, sizes, eps, d):
    x, w, dy = _case(dtype, d, sizes, d)
    # (a head of zeros has no norm without eps)
    x[..., 0] = x[..., 0] + (x[..., 0] == 0) * torch.tensor(sizes, device="cuda").to(x.dtype)
    y, _ = ops.head_norm_rotary(x, q_weight=w, eps=eps)
    v, wd = x.double(), w.double()
    eps = float(torch.tensor(eps))
    r = 1 / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + eps)
    xhat = v * r
    e = (d + 8) * 2.0 ** -24
    u, least = U[dtype], LEAST[dtype]
    _within(y, xhat * wd, (xhat * wd).abs() * (e + u) + least, "y")
    dx, _, dw, _ = ops.head_norm_rotary_backward(dy, None, x, q_weight=w, eps=eps)
    dn = dy.double() * wd
    want = r * (dn - xhat * (dn * xhat).mean(-1, keepdim=True))
    size = r * (dn.abs() + xhat.abs() * (dn * xhat).abs().mean(-1, keepdim=True))
    fits = want.abs() < float(torch.finfo(DT[dtype]).max) * 0.99
    assert float(fits.double().mean()) > 0.5
    _within(dx[fits], want[fits], (size * 4 * e + u * want.abs())[fits] + least, "dx")
    assert not bool(torch.isnan(dx.float()).any())
    many = x[..., 0].numel() + 8
    _within(dw, (dy.double() * xhat).sum((0, 1, 2)),
            (dy.double() * xhat).abs().sum((0, 1, 2)) * (e + many * 2.0 ** -24) + 1e-30, "dw")


def test_what_has_no_norm(ops):
    """Infinities, NaNs and zeros without eps: as the formula has it, and the
    heads beside them are as they were."""
    for dtype in ("f32", "bf16"):
        x, w, _ = _case(dtype, 64, (1.0, 1e30, 1.0, 1e-30), 3)
        want, _ = ops.head_norm_rotary(x, q_weight=w, eps=0.0)
        for value in (math.inf, -math.inf, math.nan):
            z = x.clone()
            z[0, 3, 1, 5] = value
            y, _ = ops.head_norm_rotary(z, q_weight=w, eps=0.0)
            assert bool(torch.isnan(y[0, 3, 1, 5]))
            mask = torch.ones(x.shape, dtype=torch.bool, device="cuda")
            mask[0, 3, 1] = False
            assert torch.equal(y[mask], want[mask])
        z = x.clone()
        z[1, 2, 0] = 0
        assert bool(torch.isnan(ops.head_norm_rotary(z, eps=0.0)[0][1, 2, 0]).all())
        assert not ops.head_norm_rotary(z)[0][1, 2, 0].any()
