"""Clipping by factors of every size: one rounding of the product, half a step of
the type (2^-24 in fp32; 2^-150 below its normal numbers), whatever the factor
is.  The values' norm in 64 bits is off by 2^-52 or so, which 1.0001 covers; a
narrower result is rounded from fp32 once more."""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import ops
    return ops


# size of the values, largest norm: ordinary ones, factors far below fp32's
# least, norms past its largest, values next to its largest and its least
SIZES = [(1.0, 0.125), (1.0, 1e-3), (1e20, 2.0 ** -70), (2e37, 1.0), (2e37, 2.0 ** -100),
         (1e30, 2.0 ** -126), (1e-38, 2.0 ** -130), (3e-42, 2.0 ** -140)]


@pytest.mark.parametrize("n", [1, 777, 300000])
@pytest.mark.parametrize("size,max_norm", SIZES, ids=str)
def test_factors(ops, size, max_norm, n):
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = (torch.randn(n, device="cuda", generator=g).clamp(-4, 4) * size).float()
    want_norm = float(x.double().norm())
    f = min(1.0, max_norm / want_norm) if want_norm else 1.0
    exact = x.double() * f
    for out in (None, [torch.empty_like(x)], "in place"):
        v = [x.clone()]
        got, norm = ops.clip_gradients(v, max_norm, out=v if out == "in place" else out)
        bound = torch.maximum(exact.abs() * 2.0 ** -24, torch.full_like(exact, 2.0 ** -150))
        assert bool(((got[0].double() - exact).abs() <= 1.0001 * bound).all())
        if want_norm < 3.4e38:
            assert abs(float(norm) - want_norm) <= want_norm * 2.0 ** -23 + 2.0 ** -149
        else:
            assert float(norm) == math.inf


@pytest.mark.parametrize("dtype,u", [(torch.float16, 2.0 ** -11), (torch.bfloat16, 2.0 ** -8)])
def test_narrow_types(ops, dtype, u):
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randn(5000, device="cuda", generator=g)
    for size, max_norm in ((1.0, 0.125), (60000.0 / 8, 2.0 ** -3)) + (
            ((2e37, 2.0 ** -10),) if dtype == torch.bfloat16 else ()):
        v = (x.clamp(-4, 4) * size).to(dtype)
        norm = float(v.double().norm())
        exact = v.double() * min(1.0, max_norm / norm)
        got, _ = ops.clip_gradients([v], max_norm)
        bound = exact.abs() * (u + 2.0 ** -24) * 1.0001 + (
            2.0 ** -25 if dtype == torch.float16 else 2.0 ** -134)
        assert bool(((got[0].double() - exact).abs() <= bound).all())
