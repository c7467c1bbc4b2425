"""The operators around a protected classifier on inputs at the ends of their
ranges: spoiled blocks and scales, values far from zero, outliers, many
images.  References are 64-bit forms; tolerances follow from the arithmetic
(fp32 sums of n terms are off by n * 2^-24 of their magnitudes at most)."""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


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


# ----------------------------------------------------------------- product

def _bytes(g, rows, cols, qtype):
    ld = -(-cols // 16) * 16
    return (30 * _randn(g, rows, ld)).to(F8[qtype])[:, :cols]


# short products, 128 x 128 tiles in one and in several ranges of k, one tile
# a compute unit, tiles that fill the card
@pytest.mark.parametrize("m,n,k,dtype", [(3, 300, 700, "f16"), (50, 300, 700, "f32"),
                                         (1280, 320, 6272, "f32"),
                                         (300, 1500, 4100, "f16"),
                                         (3601, 3540, 200, "f32"),
                                         (3601, 3540, 200, "f16"),
                                         (3601, 3540, 300, "bf16")])
@pytest.mark.parametrize("bb", [1, 128])
def test_product_spoiled_and_clean(ops, m, n, k, dtype, bb):
    """A NaN value or a NaN or infinite scale spoils its rows and columns of
    y; nothing else, not the next product's results either."""
    g = _gen(m + n + k)
    kb, nb = -(-k // 128), -(-n // bb)
    a, b = _bytes(g, m, k, "e4m3"), _bytes(g, n, k, "e4m3")
    sa = torch.rand((kb, m), device="cuda", generator=g) + 0.5
    sb = torch.rand((kb, nb), device="cuda", generator=g) + 0.5
    # (16-bit results stay finite)
    sa /= 100 * math.sqrt(k)
    sb /= 100

    def product(a, sa, b, sb):
        return ops.fp8_matmul(a, sa, b, sb, dtype=DT[dtype])
    first = product(a, sa, b, sb)
    assert bool(torch.isfinite(first).all())
    for where in ("a", "b", "sa", "sb", "sb inf"):
        args = dict(a=a, sa=sa, b=b, sb=sb)
        bad = torch.zeros((m, n), dtype=torch.bool, device="cuda")
        if where in ("a", "b"):
            v = args[where].view(torch.uint8).clone()
            v[1::37, k // 2] = 0x7f
            full = _bytes(g, *args[where].shape, "e4m3")
            full.view(torch.uint8).copy_(v)
            args[where] = full
            if where == "a":
                bad[1::37] = True
            else:
                bad[:, 1::37] = True
        elif where == "sa":
            args["sa"] = sa.clone()
            args["sa"][kb // 2, 2::37] = math.nan
            bad[2::37] = True
        else:
            v = sb.clone()
            v[:, 1::5] = math.inf if where == "sb inf" else math.nan
            args["sb"] = v
            cols = (torch.arange(n, device="cuda") // bb) % 5 == 1
            bad[:, cols] = True
        y = product(**args)
        assert torch.equal(~torch.isfinite(y), bad), where
        assert torch.equal(y[~bad], first[~bad]), where
        assert torch.equal(product(a, sa, b, sb), first), where


@pytest.mark.parametrize("m,n,k", [(3, 200, 700), (60, 200, 4096), (400, 700, 1000),
                                   (3601, 3540, 256)])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_product_of_blocks_with_outliers(ops, m, n, k, dtype):
    """Activations with a few channels hundreds of deviations out.  fp32
    results have fp32 sums; for 16-bit ones the matrix unit drops less than
    7 * 2^-13 of the largest product of every eight in a row."""
    g = _gen(m + k)
    kb = -(-k // 128)
    for far in (30.0, 300.0, 3000.0):
        x = _randn(g, m, k)
        x[:, 5::131] = far * (1 + 0.1 * _randn(g, m, len(range(5, k, 131))))
        w = _randn(g, n, k) / math.sqrt(k)
        qa, sa = ops.fp8_quantize(x)
        qb, sb = ops.fp8_quantize(w, block_rows=128)
        y = ops.fp8_matmul(qa, sa, qb, sb, dtype=DT[dtype]).double()
        want = size = drop = 0
        for i in range(kb):
            ks = slice(i * 128, min(k, i * 128 + 128))
            a, b = qa[:, ks].double(), qb[:, ks].double()
            s = sa[i].double()[:, None] * sb[i].double().repeat_interleave(128)[:n]
            want = want + (a @ b.t().contiguous()) * s
            size = size + (a.abs() @ b.abs().t().contiguous()) * s
            for j in range(0, a.shape[1], 8):
                # (the largest product is no larger than the largest of each)
                e = slice(j, j + 8)
                drop = drop + a[:, e].abs().amax(1)[:, None] * b[:, e].abs().amax(1) * s
        bound = (128 + 2 * kb + 16) * 2.0 ** -23 * size
        if dtype != "f32":
            bound = bound + 7 * 2.0 ** -13 * drop
        half = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
        off = (y - want).abs()
        bound = bound + half * want.abs() + 2.0 ** -24
        assert bool((off <= bound).all()), (far, float((off / bound).max()))


# ------------------------------------------------------------------ scores

def _check_far(ops, x, t, k, what):
    """Scores in 64 bits.  Log probabilities and entropies do not depend on
    how far from zero a row lies, so their bounds know nothing of lse: fp32
    sums of a thread's terms and the joins, exp and log of the hardware, and
    the rounding of x - max."""
    got = ops.token_scores(x, t, k)
    vocab = x.shape[1]
    v = x.double()
    m = v.amax(1, keepdim=True)
    e = torch.exp(v - m)
    s = e.sum(1, keepdim=True)
    lp = (v - m) - torch.log(s)
    h = -torch.where(e > 0, e / s * lp, 0.0).sum(1)
    lse = (m + torch.log(s))[:, 0]
    threads = 64 if vocab <= 4096 else 256 if vocab <= 16384 else 512
    rel = (vocab / threads + 64) * 2.0 ** -24 + 2.0 ** -20

    def near(a, b, bound, name):
        off = (a.double() - b).abs()
        assert bool((off <= bound).all()), (what, name, float(off.max()), a, b)
    near(got.lse, lse, rel + 2.0 ** -23 * lse.abs(), "lse")
    near(got.entropy, h, 2 * rel * (2 + h), "entropy")
    want = lp.gather(1, t.long()[:, None])[:, 0]
    near(got.logprob, want, rel + 2.0 ** -22 * want.abs(), "logprob")
    order = torch.sort(v, dim=1, descending=True, stable=True)
    k = min(k, vocab)
    assert torch.equal(got.top_ids[:, :k].long(), order[1][:, :k]), what
    want = lp.gather(1, order[1][:, :k])
    near(got.top_logprobs[:, :k], want, rel + 2.0 ** -22 * want.abs(), "top")


@pytest.mark.parametrize("vocab", [5, 100, 1000, 5000, 40000])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_token_scores_far_from_zero(ops, vocab, dtype):
    """Maxima up to fp16's largest and lowest numbers."""
    g = _gen(vocab)
    at = [-65504.0, -60000.0, -1000.0, 1000.0, 30000.0, 65504.0]
    x = torch.tensor(at, device="cuda")[:, None].repeat(2, vocab)
    x[6:] -= 4 * torch.rand((6, vocab), device="cuda", generator=g)
    x = x.to(DT[dtype])
    x = torch.cat([x.clamp(-65504, 65504), x[:2]]) if dtype != "bf16" else x
    t = torch.randint(0, vocab, (x.shape[0],), device="cuda", generator=g,
                      dtype=torch.int32)
    _check_far(ops, x, t, 5, (vocab, dtype))
    for r in range(x.shape[0]):
        _check_far(ops, x[r:r + 1], t[r:r + 1], 20, (vocab, dtype, "row", r))


# magnitudes that a type holds, up to where sums of two overflow
MAGNITUDES = [7e4, 1e6, 3e7, 1e8, 3e9, 5e9, 1e10, 1e12, 1e20, 1e30, 1e37, 3e38]


@pytest.mark.parametrize("vocab", [5, 100, 1000, 5000, 40000, 131072])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_token_scores_of_any_magnitude(ops, vocab, dtype):
    """Rows of one value, rows that spread about it by a few units of its last
    place, and ordinary rows of which a part, whole threads and workgroups
    among them, is barred by it: one wave, one workgroup, rows split over
    workgroups."""
    g = _gen(vocab)
    dt = DT[dtype]
    step = {"f32": 2.0 ** -23, "bf16": 2.0 ** -7}[dtype]
    rows = []
    for mag in MAGNITUDES:
        for v in (mag, -mag):
            rows.append(torch.full((vocab,), v, device="cuda"))
            rows.append(v * (1 + step * torch.randint(0, 4, (vocab,), device="cuda",
                                                      generator=g)))
        for part in range(3):
            x = 3 * _randn(g, vocab)
            if part == 0:
                x[torch.rand(vocab, device="cuda", generator=g) < 0.5] = -mag
            elif part == 1:
                x[vocab // 2:] = -mag
            else:
                x[:vocab - 3] = -mag
            rows.append(x)
    x = torch.stack(rows).to(dt).clamp(-3.3e38, 3.3e38)
    t = torch.randint(0, vocab, (len(rows),), device="cuda", generator=g, dtype=torch.int32)
    _check_far(ops, x, t, 5, (vocab, dtype))
    for r in range(0, len(rows), 5):
        _check_far(ops, x[r:r + 1], t[r:r + 1], 20, (vocab, dtype, "row", r))


@pytest.mark.parametrize("vocab", [1, 5, 1000, 8200, 40000])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_token_scores_backward_of_any_magnitude(ops, vocab, dtype):
    """Rows as above; probabilities follow from distances within the row, so
    their bound knows of lse only where the gradient reads it (up to 256:
    2^-17), and a row of the type's lowest value has probabilities of
    1 / vocab."""
    g = _gen(vocab)
    dt = DT[dtype]
    step = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}[dtype]
    mags = [0.5, 60.0, 250.0, 300.0, 5000.0, 3e4] + (
        [65504.0] if dtype == "f16" else MAGNITUDES + [torch.finfo(dt).max])
    rows = []
    for mag in mags:
        for v in (mag, -mag):
            rows.append(torch.full((vocab,), v, device="cuda", dtype=torch.float64))
            rows.append(v * (1 - step * torch.randint(0, 4, (vocab,), device="cuda",
                                                      generator=g).double()))
            rows.append(torch.where(torch.rand(vocab, device="cuda", generator=g) < 0.3,
                                    -math.inf, v))
        x = 3 * _randn(g, vocab).double()
        x[vocab // 2:] = -mag
        rows.append(x)
    x = torch.stack(rows).to(dt)
    n = len(rows)
    t = torch.randint(0, vocab, (n,), device="cuda", generator=g, dtype=torch.int32)
    t[::5] = -1
    gl, glp, gh = (_randn(g, n) for _ in range(3))
    r = ops.token_scores(x, t)
    got = ops.token_scores_backward(x, t, r.lse, r.entropy, gl, glp, gh)
    v = x.double()
    m = v.amax(1, keepdim=True)
    empty = m == -math.inf
    m = torch.where(empty, 0.0, m)
    e = torch.exp(v - m)
    s = torch.where(empty, 1.0, e.sum(1, keepdim=True))
    lp = (v - m) - torch.log(s)
    p = e / s
    inner = torch.where(p > 0, lp, 0.0)
    h = -(p * inner).sum(1, keepdim=True)
    gl, gh = gl.double()[:, None], gh.double()[:, None]
    glp = torch.where((t >= 0)[:, None] & ~empty, glp.double()[:, None], 0.0)
    one = torch.zeros_like(p).scatter_(1, t.clamp(min=0).long()[:, None], 1.0)
    want = p * (gl - glp - gh * (inner + h)) + one * glp
    size = (p * (gl.abs() + glp.abs() + gh.abs() * ((inner + h).abs() + h + 1)) *
            (1 + inner.abs()) + one * glp.abs())
    rel = (vocab / 256 + 64) * 2.0 ** -24 + 2.0 ** -19
    rel = torch.where((m + torch.log(s)).abs() <= 257, rel + 2.0 ** -17, rel)
    half = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}[dtype]
    off = (got.double() - want).abs()
    bound = rel * size + half * want.abs() + 2.0 ** -25
    assert bool((off <= bound).all()), float((off / bound).max())
    assert torch.equal(ops.token_scores_backward(x, t, r.lse, r.entropy, gl[:, 0].float(),
                                                 torch.where(t >= 0, glp[:, 0], 0.0).float(),
                                                 gh[:, 0].float(), out=x), got)


# -------------------------------------------------------------- group norm

def _norm_ref(x, dy, groups, gamma, beta):
    """y, mean, rstd, dx, dgamma, dbeta in 64 bits, with the magnitudes that
    their sums are of; act is the SiLU."""
    n, hw, c = x.shape
    sh = (n, hw, groups, c // groups)
    v = x.double().view(sh)
    var, mean = torch.var_mean(v, (1, 3), correction=0, keepdim=True)
    rstd = 1 / torch.sqrt(var + 1e-5)
    xhat = ((v - mean) * rstd).view(n, hw, c)
    z = xhat * gamma.double() + beta.double()
    s = torch.sigmoid(z)
    dz = dy.double() * (s + z * s * (1 - s))
    dn = (dz * gamma.double()).view(sh)
    xg = xhat.view(sh)
    m1, m2 = dn.mean((1, 3), keepdim=True), (dn * xg).mean((1, 3), keepdim=True)
    dx = ((dn - m1 - xg * m2) * rstd).view(n, hw, c)
    size = ((dn.abs() + dn.abs().mean((1, 3), keepdim=True) + xg.abs() *
             (dn * xg).abs().mean((1, 3), keepdim=True)) * rstd).view(n, hw, c)
    return dict(y=z * s, mean=mean[:, 0, :, 0], rstd=rstd[:, 0, :, 0], dx=dx,
                dgamma=(dz * xhat).sum((0, 1)), dbeta=dz.sum((0, 1)), size=size,
                z=z, xhat=xhat, sg=(dz * xhat).abs().sum((0, 1)),
                sb=dz.abs().sum((0, 1)))


# workgroups of one image's slabs and of chunks, of more than 2^20 in all
@pytest.mark.parametrize("n,hw,c,groups", [(4093, 1, 512, 32), (4094, 1, 16, 4),
                                           (4100, 4, 24, 3), (10000, 9, 64, 8),
                                           (4097, 2, 1028, 1), (1100000, 1, 8, 2),
                                           (530000, 1, 1028, 1)], ids=str)
def test_group_norm_of_many_images(ops, n, hw, c, groups):
    g = _gen(n)
    x, dy = _randn(g, n, hw, c), _randn(g, n, hw, c)
    gamma, beta = 0.5 + torch.rand(c, device="cuda", generator=g), 0.3 * _randn(g, c)
    y, mean, rstd = ops.group_norm(x, groups, gamma, beta, act="silu")
    dx, _, dgamma, dbeta = ops.group_norm_backward(dy, x, mean, rstd, groups, gamma, beta,
                                                   act="silu")
    # an image's sums are of hw * c / groups terms (and 24 more operations);
    # silu' is at most 1.1 and moves by at most 0.5 a unit of z
    u = (hw * c / groups + 24) * 2.0 ** -24
    totals = {k: 0 for k in ("dgamma", "dbeta", "sg", "sb")}
    for i in range(0, n, 100000):
        part = slice(i, i + 100000)
        w = _norm_ref(x[part], dy[part], groups, gamma, beta)
        for k in totals:
            totals[k] = totals[k] + w[k]
        spread = 1 / w["rstd"]
        for got, k, bound in [
                (mean, "mean", u * (w["mean"].abs() + spread)), (rstd, "rstd", u * w["rstd"]),
                (y, "y", 2 * u * (1 + w["xhat"].abs() + w["z"].abs())),
                (dx, "dx", 4 * u * w["size"] * (1 + w["z"].abs()) ** 2)]:
            off = (got[part].double() - w[k]).abs()
            assert bool((off <= bound).all()), (k, i, float((off / bound).max()))
    u = (n * hw / 64 + 64) * 2.0 ** -24
    for got, k, s in ((dgamma, "dgamma", "sg"), (dbeta, "dbeta", "sb")):
        off = (got.double() - totals[k]).abs()
        assert bool((off <= 4 * u * totals[s]).all()), (k, float((off / totals[s]).max()))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("n,hw,c,groups", [(4, 12544, 8, 1), (1, 50176, 8, 1), (1, 50176, 24, 3),
                                           (3, 9000, 32, 4)], ids=str)
def test_group_norm_outliers(ops, n, hw, c, groups, dtype):
    """Pixels up to 1000 deviations out, the first one of the map among them:
    chunks are summed in 64 bits and joined so, and rounded a few times."""
    for far in (0.0, 10.0, 100.0, 1000.0, -30000.0):
        x = _randn(_gen(hw), n, hw, c)
        if far:
            x[:, 0] = far
            x[:, hw // 3, 1] = -far
            x[:, -1] = far
        x = x.to(DT[dtype])
        _, mean, rstd = ops.group_norm(x, groups)
        v = x.double().view(n, hw, groups, c // groups)
        var, want = torch.var_mean(v, (1, 3), correction=0)
        wr = 1 / torch.sqrt(var + 1e-5)
        off = (rstd.double() / wr - 1).abs().max()
        assert float(off) <= 16 * 2.0 ** -24, (far, float(off))
        off = ((mean.double() - want).abs() * wr).max()
        assert float(off) <= 4 * 2.0 ** -24, (far, float(off))


# held by a workgroup, and beyond one: a group of its own, several chunks
@pytest.mark.parametrize("n,hw,c,groups", [(3, 1, 64, 4), (130, 1, 16, 2), (3, 1, 1028, 1),
                                           (3, 9000, 32, 8)], ids=str)
def test_group_norm_gradient_sums_that_cancel(ops, n, hw, c, groups):
    """dbeta and dgamma over images whose parts cancel: 2^24, 1 and -2^24 of
    one pixel, all of them exact, of which fp32 sums leave 0."""
    x = _randn(_gen(c), 1, hw, c).repeat(n, 1, 1)
    dy = torch.zeros_like(x)
    dy[0, 0], dy[1, 0], dy[-1, 0] = 2.0 ** 24, 1.0, -2.0 ** 24
    _, mean, rstd = ops.group_norm(x, groups)
    _, _, dgamma, dbeta = ops.group_norm_backward(dy, x, mean, rstd, groups)
    assert bool((dbeta == 1).all())
    per = c // groups
    want = (x[0, 0].double() - mean[0].double().repeat_interleave(per)) * \
        rstd[0].double().repeat_interleave(per)
    # (the difference and the product are rounded once each)
    assert bool(((dgamma.double() - want).abs() <= 2.0 ** -22 * (1 + want.abs())).all())


@pytest.mark.parametrize("hw,c", [(16, 64), (16, 12), (30000, 24), (1, 1028)])
def test_group_norm_of_channels_whose_means_cancel(ops, hw, c):
    """Channels of 2^20, 1, -2^20 and 0: their sums are exact, and the group's
    mean is a quarter."""
    x = torch.tensor([2.0 ** 20, 1.0, -2.0 ** 20, 0.0], device="cuda").repeat(c // 4)
    x = x.expand(2, hw, c).contiguous()
    for groups in {1, c // 4}:
        y, mean, rstd = ops.group_norm(x, groups)
        assert bool(((mean - 0.25).abs() <= 2.0 ** -24).all()), mean
        want = 1 / math.sqrt((2.0 ** 41 + 1) / 4 - 1 / 16 + 1e-5)
        assert bool(((rstd.double() / want - 1).abs() <= 2.0 ** -21).all())


# ------------------------------------------------------ torch's own accounts

def _calls(ops):
    """(call, tensors it takes by name, names of its outputs) of each entry
    point; outputs are given."""
    e = torch.empty
    x = torch.randn((2, 4, 8), device="cuda")
    m = torch.randn((4, 32), device="cuda")
    q, s = ops.fp8_quantize(m)
    t = torch.tensor([1, 2, 3, 4], device="cuda", dtype=torch.int32)
    _, mean, rstd = ops.group_norm(x, 2)
    r = ops.token_scores(m, t, 2)
    g = torch.ones(4, device="cuda")
    f = dict(device="cuda")
    return [
        (lambda x, gamma, beta, residual, y, mean, rstd: ops.group_norm(
            x, 2, gamma, beta, residual, out=(y, mean, rstd)),
         dict(x=x, gamma=e(8, **f), beta=e(8, **f), residual=x.clone(), y=x.clone(),
              mean=mean.clone(), rstd=rstd.clone()), ("y", "mean", "rstd")),
        (lambda dy, x, mean, rstd, gamma, beta, residual, dx, dr, dg, db:
         ops.group_norm_backward(dy, x, mean, rstd, 2, gamma, beta, residual,
                                 out=(dx, dr, dg, db)),
         dict(dy=x.clone(), x=x, mean=mean, rstd=rstd, gamma=e(8, **f), beta=e(8, **f),
              residual=x.clone(), dx=x.clone(), dr=x.clone(), dg=e(8, **f),
              db=e(8, **f)), ("dx", "dr", "dg", "db")),
        (lambda x, q, s: ops.fp8_quantize(x, out=(q, s)),
         dict(x=m, q=q.clone(), s=s.clone()), ("q", "s")),
        (lambda sa, sb, bias, out: ops.fp8_matmul(q, sa, q, sb, bias, out=out),
         dict(sa=s, sb=s.clone(), bias=g, out=e((4, 4), **f)), ("out",)),
        (lambda x, lse, entropy, logprob, rank, ids, tops: ops.token_scores(
            x, t, 2, out=ops.TokenScores(lse, entropy, logprob, rank, ids, tops)),
         dict(x=m, lse=r.lse.clone(), entropy=r.entropy.clone(), logprob=r.logprob.clone(),
              rank=r.rank.clone(), ids=r.top_ids.clone(), tops=r.top_logprobs.clone()),
         ("lse", "entropy", "logprob", "rank", "ids", "tops")),
        (lambda x, lse, entropy, g1, g2, g3, out: ops.token_scores_backward(
            x, t, lse, entropy, g1, g2, g3, out=out),
         dict(x=m, lse=r.lse, entropy=r.entropy, g1=g, g2=g.clone(), g3=g.clone(),
              out=m.clone()), ("out",)),
    ]


def test_tensors_that_require_grad_are_refused(ops):
    """Results carry no graph, so a gradient would be lost silently."""
    for i, (call, args, _) in enumerate(_calls(ops)):
        call(**args)
        for name, v in args.items():
            if v.dtype != torch.float32:
                continue
            with_grad = dict(args, **{name: v.clone().requires_grad_()})
            with pytest.raises(ValueError, match="grad"):
                call(**with_grad)
                raise AssertionError((i, name))
            with torch.no_grad():
                call(**with_grad)
            call(**dict(with_grad, **{name: with_grad[name].detach()}))


def test_given_outputs_count_as_changed(ops):
    """torch's version of a tensor rises when it is written, so a backward
    pass that saved its values refuses them; other tensors' do not."""
    for i, (call, args, outs) in enumerate(_calls(ops)):
        before = {name: v._version for name, v in args.items()}
        call(**args)
        for name, v in args.items():
            assert (v._version > before[name]) == (name in outs), (i, name)
    # in place, where a saved value is lost
    w = torch.ones((2, 4, 8), device="cuda", requires_grad=True)
    z = torch.randn((2, 4, 8), device="cuda")
    loss = (w * z).sum()
    ops.group_norm(z, 2, out=(z, torch.empty((2, 2), device="cuda"),
                              torch.empty((2, 2), device="cuda")))
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():
        m = torch.randn((4, 32), device="cuda")
        r = ops.token_scores(m)
        ops.token_scores(m, out=r)
