"""Norms of heads with rotations, their gradients, and clipping, against the
formulas in 64 bits.

Tolerances: a head's mean square is a sum of d terms in fp32 (d 2^-24 of it at
most), its root and reciprocal two roundings; an angle is good to 2^-21; a
result is rounded once (half a step u of its type).
"""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}
TINY = {"f32": 0.0, "f16": 2.0 ** -25, "bf16": 0.0}     # half a subnormal step


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
    over = ~((got - want).abs() <= bound)
    if bool(over.any()):
        i = int(((got - want).abs() / bound).nan_to_num(1e300).masked_fill(~over, 0).argmax())
        raise AssertionError("%s: %d of %d off, worst at %d: %.9g for %.9g, bound %.3g" % (
            what, int(over.sum()), over.numel(), i, got.flatten()[i],
            want.flatten()[i], bound.flatten()[i]))


def _order(d, turned, interleaved):
    """(first, second) indices of the turned pairs."""
    p = torch.arange(turned, device="cuda")
    return (2 * p, 2 * p + 1) if interleaved else (p, p + turned)


def _angles(positions, frequencies, axes, b):
    axis = torch.repeat_interleave(torch.arange(len(axes)), torch.tensor(axes)).cuda()
    a = positions.double()[..., axis] * frequencies.double()
    return (a if a.dim() == 3 else a[None].expand(b, -1, -1))[:, :, None]


def _turn(z, angles, pairs, back=False):
    y = z.clone()
    c, s = torch.cos(angles), torch.sin(angles) * (-1 if back else 1)
    a, b = z[..., pairs[0]], z[..., pairs[1]]
    y[..., pairs[0]], y[..., pairs[1]] = a * c - b * s, a * s + b * c
    return y


# b, tokens, q heads, k heads, head size, axes, interleaved, positions of their
# own: whole vectors, odd numbers of pairs, values that are not turned, no
# keys, no rotation, heads wider than a wave's vectors
CASES = [(2, 49, 8, 8, 64, (16, 16), False, False),
         (1, 1, 1, 0, 2, (1,), False, False), (3, 5, 3, 1, 10, (2, 1), False, True),
         (2, 17, 4, 2, 80, (16, 12, 12), False, False), (1, 33, 2, 2, 40, (7,), False, True),
         (2, 9, 5, 5, 96, (16, 16, 16), True, True), (1, 3, 2, 1, 6, (3,), True, False),
         (1, 8, 2, 1, 64, (), False, False), (1, 4, 3, 2, 512, (128, 64), False, False),
         (2, 3, 1, 1, 264, (64, 64), True, False), (1, 7, 16, 16, 128, (8, 0, 24), False, False),
         (1, 2100, 1, 1, 32, (4, 4, 4, 4), False, False)]


@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("types", [("f32", "f32"), ("f32", "f16"), ("f32", "bf16"),
                                   ("f16", "f16"), ("bf16", "bf16")], ids=str)
@pytest.mark.parametrize("case", CASES, ids=str)
def test_head_norm_rotary(ops, case, types, norm):
    b, t, hq, hk, d, axes, inter, own = case
    dt, to = DT[types[0]], DT[types[1]]
    u = U[types[1]]
    if not norm and types[0] != types[1]:
        pytest.skip("one type is enough")
    g = _gen(7)
    both = (1.5 * _randn(g, b, t, hq + hk, d)).to(dt)
    x = {"q": both[:, :, :hq]}
    if hk:
        x["k"] = both[:, :, hq:]
    w = {n: 1 + 0.3 * _randn(g, d) for n in "qk"}
    n_axes, turned = len(axes), sum(axes)
    pos = torch.randint(-50, 5000, (b, t, n_axes) if own else (t, n_axes), device="cuda",
                        generator=g, dtype=torch.int32)
    freq = torch.rand(turned, device="cuda", generator=g)
    kw = dict(q_weight=w["q"], k_weight=w["k"], axes=axes, interleaved=inter, norm=norm, eps=1e-5)
    if axes:
        kw.update(positions=pos, frequencies=freq)
    got = dict(zip("qk", ops.head_norm_rotary(x["q"], x.get("k"), dtype=to, **kw)))
    dy = {n: _randn(g, *x[n].shape).to(to) for n in x}
    r = ops.head_norm_rotary_backward(dy["q"], dy.get("k"), x["q"], x.get("k"), **kw)
    grads = {"q": (r[0], r[2]), "k": (r[1], r[3])}
    if not hk:
        assert got["k"] is None and r[1] is None and r[3] is None
    pairs = _order(d, turned, inter)
    angles = _angles(pos, freq, axes, b) if axes else None
    e = (d + 8) * 2.0 ** -24           # of a normed value
    for n in x:
        v, wd = x[n].double(), w[n].double()
        r = 1 / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + 1e-5) if norm \
            else torch.ones_like(v[..., :1])
        z = v * r * wd
        y, size = z, z.abs()
        if axes:
            y = _turn(z, angles, pairs)
            size = size.clone()
            size[..., pairs[0]] = size[..., pairs[1]] = (z[..., pairs[0]].abs()
                                                         + z[..., pairs[1]].abs())
        _within(got[n], y, size * (e + 2.0 ** -21) + u * y.abs() + TINY[types[1]], n)
        dz, dsize = dy[n].double(), dy[n].double().abs()
        if axes:
            dsize = dsize.clone()
            dsize[..., pairs[0]] = dsize[..., pairs[1]] = (dz[..., pairs[0]].abs()
                                                           + dz[..., pairs[1]].abs())
            dz = _turn(dz, angles, pairs, back=True)
        xhat = v * r
        dw = (dz * xhat).sum((0, 1, 2))
        many = b * t * x[n].shape[2] + 8
        _within(grads[n][1], dw, (dsize * xhat.abs()).sum((0, 1, 2)) *
                (e + 2.0 ** -21 + many * 2.0 ** -24) + 1e-30, "d%s_weight" % n)
        dn, an = dz * wd, dsize * wd.abs()
        dx, size = dn, an
        if norm:
            dx = r * (dn - xhat * (dn * xhat).mean(-1, keepdim=True))
            size = r * (an + xhat.abs() * (an * xhat.abs()).mean(-1, keepdim=True))
        _within(grads[n][0], dx, size * (4 * e + 2.0 ** -20) + U[types[0]] * dx.abs()
                + TINY[types[0]], "d" + n)


def test_far_positions(ops):
    """An angle of two thousand million steps is as good as a near one."""
    d = 64
    pos = torch.tensor([[2 ** 31 - 1], [-2 ** 31], [2 ** 24 + 1], [0]], dtype=torch.int32,
                       device="cuda")
    freq = torch.tensor([1.0 / (1 + i) for i in range(d // 2)], device="cuda")
    x = torch.ones((1, 4, 1, d), device="cuda")
    y, _ = ops.head_norm_rotary(x, positions=pos, frequencies=freq, axes=(d // 2,), norm=False)
    a = pos.double()[None, :, None] * freq.double()
    want = torch.cat([torch.cos(a) - torch.sin(a), torch.sin(a) + torch.cos(a)], -1)
    assert float((y.double() - want).abs().max()) <= 2 * 2.0 ** -21 + 2.0 ** -23


def test_in_place(ops):
    g = _gen(3)
    both = _randn(g, 2, 31, 6, 64).to(torch.bfloat16)
    pos = ops.grid_positions(31)
    freq = ops.rotary_frequencies((32,))
    kw = dict(positions=pos, frequencies=freq, axes=(32,))
    q, k = both[:, :, :4], both[:, :, 4:]
    want = ops.head_norm_rotary(q, k, **kw)
    dq, dk = torch.randn_like(want[0]), torch.randn_like(want[1])
    grads = ops.head_norm_rotary_backward(dq, dk, q, k, **kw)
    again = ops.head_norm_rotary_backward(dq, dk, q, k, out=(dq, dk, None, None), **kw)
    assert again[2] is None and again[3] is None
    assert torch.equal(dq, grads[0]) and torch.equal(dk, grads[1])
    ops.head_norm_rotary(q, k, out=(q, k), **kw)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])


# ---------------------------------------------------------------- clipping

def _check_clip(ops, grads, max_norm, place):
    want = math.sqrt(sum(float((v.double() ** 2).sum()) for v in grads))
    f = max_norm / want if want > max_norm else 1.0
    before = [v.clone() for v in grads]
    out = {"new": None, "given": [torch.full_like(v, 7) for v in grads], "in place": grads}[place]
    got, norm = ops.clip_gradients(grads, max_norm, out=out)
    assert abs(float(norm) - want) <= want * 2.0 ** -23
    for x, y, b in zip(before, got, grads):
        u = {4: 2.0 ** -24, 2: 2.0 ** -11 if x.dtype == torch.float16 else 2.0 ** -8}[
            x.element_size()]
        exact = x.double() * f
        tiny = 2.0 ** -25 if x.dtype == torch.float16 else 2.0 ** -149
        assert bool(((y.double() - exact).abs() <= exact.abs() * (2.0 ** -23 + u) + tiny).all())
        if place != "in place":
            assert torch.equal(b, x)
        if f == 1.0:
            assert torch.equal(y, x)


@pytest.mark.parametrize("place", ["new", "given", "in place"])
@pytest.mark.parametrize("clipped", [True, False])
def test_clip(ops, clipped, place):
    """Empty tensors, single values, odd sizes, more tensors than a launch's
    table, every type, addresses of one element, transposed ones."""
    g = _gen(11)
    sizes = [0, 1, 7, 16384, 16385, 3 * 16384 + 5, 100003, 0] + [13 + i for i in range(230)]
    grads = []
    for i, n in enumerate(sizes):
        t = list(DT.values())[i % 3]
        store = _randn(g, n + 1).to(t)
        grads.append(store[1:] if i % 2 else store[:n])
    grads.append(_randn(g, 33, 65).t())
    grads.append(_randn(g, 1).reshape(()))
    norm = math.sqrt(sum(sizes))
    _check_clip(ops, grads, norm * (0.1 if clipped else 10), place)


def test_clip_large_values(ops):
    """fp32 values whose squares overflow fp32, and a norm that is infinite or
    NaN: values stay as they are."""
    g = _gen(5)
    a = _randn(g, 1000) * 1e30
    _check_clip(ops, [a], 1.0, "new")
    for bad in (math.inf, math.nan):
        x = _randn(g, 5000)
        x[77] = bad
        out, norm = ops.clip_gradients([x, _randn(g, 3)], 1e-3)
        assert not math.isfinite(float(norm))
        assert torch.equal(out[0].nan_to_num(9.0), x.nan_to_num(9.0))
    x = torch.zeros(10, device="cuda")
    out, norm = ops.clip_gradients([x], 0.0)
    assert float(norm) == 0 and torch.equal(out[0], x)
    out, norm = ops.clip_gradients([x + 1], 0.0)
    assert torch.equal(out[0], x)
    out, norm = ops.clip_gradients([x + 1], math.inf)
    assert torch.equal(out[0], x + 1)
