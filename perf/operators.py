"""The operators around a protected classifier, as timed cases.

Group norm with an activation on channels-last maps, the 8-bit quantiser and
the 8-bit block-scaled product, and the scores of given classes or tokens
(log probability, entropy, rank, top alternatives), each with its backward
pass where it has one.  Sizes are those of the repository's networks (maps
from 7x7 to 224x224, classifier layers of 1000 classes, 25088 x 4096 and
4096 x 4096 filters, 1x1 layers) and generic sizes of larger vocabularies.

The plain forms compute in 32 bits with elementary torch operations.
"""

import math

import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
F8_MAX = {"e4m3": 448.0, "e5m2": 57344.0}
BLOCK = 128
EPS = 1e-5
# The largest pass that is drawn: elements of a map, of a quantised matrix
# and of a batch of logits, and multiply-adds of a product.
MOST_MAP = 32 * 112 * 112 * 128
MOST_QUANT = 8192 * 4096
MOST_LOGITS = 2048 * 131072
MOST_MACS = 8192 * 4096 * 8192


# ------------------------------------------------------------------- cases

def _gn(name, dtype, n, h, w, c, groups, act, residual=False, carry=False,
        backward=False):
    return dict(name=name, op="group_norm", dtype=dtype, n=n, h=h, w=w, c=c,
                groups=groups, act=act, residual=residual, carry=carry,
                backward=backward)


def _quant(name, dtype, rows, cols, qtype, block_rows=1, transpose=False):
    return dict(name=name, op="quantize", dtype=dtype, rows=rows, cols=cols,
                qtype=qtype, block_rows=block_rows, transpose=transpose)


def _mm(name, dtype, m, n, k, a="e4m3", b_block=128, bias=True, act="none"):
    return dict(name=name, op="matmul", dtype=dtype, m=m, n=n, k=k, a=a,
                b_block=b_block, bias=bias, act=act)


def _scores(name, dtype, rows, vocab, pad=0, top_k=0, masked=False,
            backward=False):
    return dict(name=name, op="scores", dtype=dtype, rows=rows, vocab=vocab,
                pad=pad, top_k=top_k, masked=masked, backward=backward)


def listed():
    return [
        # One image's last feature map, in a serving call: latency.
        _gn("gn_f32_b1_7x7_512", "f32", 1, 7, 7, 512, 32, "relu"),
        # The norm that closes a residual block of a protected network, at
        # the evaluation batch.
        _gn("gn_f16_b64_56x56_64", "f16", 64, 56, 56, 64, 16, "relu",
            residual=True, carry=True),
        # A training step's gradient on the large early maps.
        _gn("gn_grad_bf16_b32_112x112_128", "bf16", 32, 112, 112, 128, 32,
            "silu", backward=True),
        # The activations of a 1x1 layer on 7x7 maps (rows: pixels), whose
        # width is no whole number of blocks.
        _quant("quant_f16_6272x320", "f16", 6272, 320, "e4m3"),
        # The gradient of a wide layer laid out for its weight gradient.
        _quant("quant_bf16_8192x4096_t", "bf16", 8192, 4096, "e5m2",
               transpose=True),
        # The classifier of a protected network on one image: 1000 classes
        # and the checksum neuron.
        _mm("mm_f16_m1_n1001_k4096", "f16", 1, 1001, 4096),
        # The first hidden layer of the largest network's classifier at its
        # evaluation batch: the filters are read once.
        _mm("mm_f16_m32_n4096_k25088", "f16", 32, 4096, 25088, act="relu"),
        # The weight gradient of the 1x1 layer on 7x7 maps: few outputs, a
        # long sum over the batch's pixels.
        _mm("mm_wgrad_f32_m1280_n320_k6272", "f32", 1280, 320, 6272,
            a="e5m2", b_block=1, bias=False),
        # A wide layer on a training batch.
        _mm("mm_bf16_m8192_n4096_k8192", "bf16", 8192, 4096, 8192),
        # The answers of a protected classifier on its evaluation batch
        # (the row's last value is the checksum and takes no part).
        _scores("scores_f32_128x1000", "f32", 128, 1000, pad=1, top_k=5),
        # A batch of positions over a large vocabulary, some tokens barred.
        _scores("scores_bf16_2048x131072", "bf16", 2048, 131072, top_k=20,
                masked=True),
        # The gradient of such scores, over an odd vocabulary.
        _scores("scores_grad_f16_4096x32001", "f16", 4096, 32001,
                backward=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice([_draw_gn, _draw_gn, _draw_quant, _draw_mm,
                           _draw_mm, _draw_scores, _draw_scores])
        case = kind(rng)
        if _size(case) <= 1.0:
            del case["name"]
            return case


def _size(case):
    """The case's size against the largest of its kind."""
    if case["op"] == "group_norm":
        return case["n"] * case["h"] * case["w"] * case["c"] / MOST_MAP
    if case["op"] == "quantize":
        return case["rows"] * case["cols"] / MOST_QUANT
    if case["op"] == "matmul":
        return max(case["m"] * case["n"] * case["k"] / MOST_MACS,
                   case["n"] * case["k"] / (25088 * 4096))
    return case["rows"] * case["vocab"] / MOST_LOGITS


def _draw_gn(rng):
    groups = rng.choice([1, 4, 8, 16, 32])
    per = _log(rng, 1, 64)
    h = _log(rng, 1, 224)
    w = rng.choice([h, h, max(1, h + rng.randint(-5, 5))])
    return _gn("", rng.choice(["f32", "f16", "bf16"]), _log(rng, 1, 128), h,
               w, max(2, groups * per), groups,
               rng.choice(["none", "relu", "silu"]),
               residual=rng.random() < 0.4, carry=rng.random() < 0.4,
               backward=rng.random() < 0.5)


def _draw_quant(rng):
    return _quant("", rng.choice(["f32", "f16", "bf16"]), _log(rng, 1, 32768),
                  _log(rng, 10, 25088), rng.choice(["e4m3", "e4m3", "e5m2"]),
                  block_rows=rng.choice([1, 1, 128]),
                  transpose=rng.random() < 0.5)


def _draw_mm(rng):
    m, n, k = _log(rng, 1, 16384), _log(rng, 10, 8192), _log(rng, 32, 25088)
    if rng.random() < 0.3:
        return _mm("", "f32", m, n, k, a="e5m2", b_block=1, bias=False)
    return _mm("", rng.choice(["f32", "f16", "bf16"]), m, n, k,
               a=rng.choice(["e4m3", "e4m3", "e5m2"]),
               bias=rng.random() < 0.5,
               act=rng.choice(["none", "relu", "silu"]))


def _draw_scores(rng):
    return _scores("", rng.choice(["f32", "f16", "bf16"]),
                   _log(rng, 1, 16384), _log(rng, 10, 131072),
                   pad=rng.choice([0, 0, 1, 8]),
                   top_k=rng.choice([0, 1, 5, 20]),
                   masked=rng.random() < 0.4, backward=rng.random() < 0.4)


def work(case):
    e = torch.empty((), dtype=DT[case["dtype"]]).element_size()
    if case["op"] == "group_norm":
        x = case["n"] * case["h"] * case["w"] * case["c"]
        res = int(case["residual"])
        if case["backward"]:
            return {"bytes": x * e * (3 + 2 * res) + 16 * case["c"]
                    + 8 * case["n"] * case["groups"], "flops": 16 * x}
        return {"bytes": x * e * (2 + res) + 8 * case["c"]
                + 8 * case["n"] * case["groups"], "flops": 8 * x}
    if case["op"] == "quantize":
        x = case["rows"] * case["cols"]
        scales = x // (BLOCK * case["block_rows"]) + 1
        return {"bytes": x * (e + 1) + 4 * scales, "flops": 2 * x}
    if case["op"] == "matmul":
        m, n, k = case["m"], case["n"], case["k"]
        kb = -(-k // BLOCK)
        return {"bytes": (m + n) * k + m * n * e
                + 4 * kb * (m + -(-n // case["b_block"]))
                + (4 * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    x = case["rows"] * case["vocab"]
    if case["backward"]:
        return {"bytes": 2 * x * e + 20 * case["rows"], "flops": 6 * x}
    return {"bytes": x * e + case["rows"] * (20 + 8 * case["top_k"]),
            "flops": 5 * x}


# ------------------------------------------------------------------ inputs

def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _rand(g, *shape):
    return torch.rand(shape, device="cuda", generator=g)


def prepare(case, seed):
    g = _gen(seed)
    return {"group_norm": _prepare_gn, "quantize": _prepare_quant,
            "matmul": _prepare_mm, "scores": _prepare_scores}[case["op"]](
                case, g)


def _prepare_gn(case, g):
    dt = DT[case["dtype"]]
    shape = (case["n"], case["h"], case["w"], case["c"])
    # what a convolution gives: channels of their own mean and spread
    x = _randn(g, *shape)
    x *= 0.5 + _rand(g, case["c"])
    x += _randn(g, case["c"])
    if case["carry"]:
        x[..., -1] = 3.0 * x[..., -1].abs()
    s = {"case": case, "x": x.to(dt),
         "gamma": 0.5 + _rand(g, case["c"]), "beta": 0.2 * _randn(g, case["c"]),
         "residual": (_randn(g, *shape).relu_().to(dt) if case["residual"]
                      else None)}
    if case["backward"]:
        s["dy"] = _randn(g, *shape).to(dt)
        xg = s["x"].float().reshape(case["n"], -1, case["groups"],
                                    case["c"] // case["groups"])
        s["mean"], s["rstd"] = _stats(xg, case["carry"])
    return s


def _blocks(rows, block_rows):
    return -(-rows // block_rows)


def _quantize(x, qtype, block_rows):
    """q and the scales [blocks of columns][blocks of rows] of a matrix: the
    largest magnitude of a block becomes the type's largest value."""
    rows, cols = x.shape
    kb, rb = _blocks(cols, BLOCK), _blocks(rows, block_rows)
    x = x.float()
    t = torch.nn.functional.pad(x.abs(), (0, kb * BLOCK - cols, 0,
                                          rb * block_rows - rows))
    amax = t.reshape(rb, block_rows, kb, BLOCK).amax((1, 3)).t()
    amax = torch.clamp(amax, min=2.0 ** -100)
    scales = (amax / F8_MAX[qtype]).contiguous()
    inv = F8_MAX[qtype] / amax
    q = _padded(rows, cols, F8[qtype])
    q.copy_((x * _spread(inv, rows, cols, block_rows)).to(F8[qtype]))
    return q, scales


def _padded(rows, cols, dtype):
    """A matrix whose rows begin at multiples of 16 elements."""
    return torch.empty((rows, -(-cols // 16) * 16), dtype=dtype,
                       device="cuda")[:, :cols]


def _spread(s, rows, cols, block_rows):
    """Scales [blocks of columns][blocks of rows] for every element."""
    s = s.t().repeat_interleave(BLOCK, 1)[:, :cols]
    return s if block_rows == 1 else s.repeat_interleave(block_rows,
                                                         0)[:rows]


def _prepare_quant(case, g):
    x = _randn(g, case["rows"], case["cols"])
    x *= torch.exp(_randn(g, case["rows"], 1))
    if case["qtype"] == "e4m3" and case["block_rows"] == 1:
        x.relu_()                       # activations
    return {"case": case, "x": x.to(DT[case["dtype"]])}


def _prepare_mm(case, g):
    m, n, k = case["m"], case["n"], case["k"]
    a = _randn(g, m, k) * torch.exp(0.5 * _randn(g, m, 1))
    if case["a"] == "e4m3":
        a.relu_()
    a, sa = _quantize(a, case["a"], 1)
    w = _randn(g, n, k) * (math.sqrt(2.0 / k) if case["b_block"] == BLOCK
                           else 1.0)
    b, sb = _quantize(w, "e4m3", case["b_block"])
    return {"case": case, "a": a, "sa": sa, "b": b, "sb": sb,
            "bias": 0.1 * _randn(g, n) if case["bias"] else None}


def _prepare_scores(case, g):
    rows, vocab = case["rows"], case["vocab"]
    x = 2.5 * _randn(g, rows, vocab + case["pad"])
    if case["masked"]:
        x.masked_fill_(_rand(g, 1, vocab + case["pad"]) < 0.1, -math.inf)
        if rows > 4:
            x[rows // 2] = -math.inf    # a row that allows nothing
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=g,
                      dtype=torch.int32)
    t[::7] = -1                         # positions without a target
    s = {"case": case, "logits": x.to(DT[case["dtype"]])[:, :vocab],
         "targets": t}
    if case["backward"]:
        r = _scores_plain(s["logits"], t, 0)
        s["lse"], s["entropy"] = r["lse"], r["entropy"]
        # 16-bit gradients come of a scaled loss
        scale = 4096.0 if case["dtype"] == "f16" else 1.0
        s["g_logprob"] = -scale * _rand(g, rows)
        s["g_entropy"] = 0.01 * scale * _rand(g, rows)
    return s


# ------------------------------------------------------------- plain forms

def _stats(xg, carry):
    """mean and rstd [n, groups] of [n, pixels, groups, channels]."""
    count = torch.full((xg.shape[2],), float(xg.shape[1] * xg.shape[3]),
                       dtype=xg.dtype, device=xg.device)
    mean, mask = xg, None
    if carry:
        mask = torch.ones(xg.shape[2:], dtype=xg.dtype, device=xg.device)
        mask[-1, -1] = 0
        count[-1] -= xg.shape[1]
        count.clamp_(min=1)
        mean = xg * mask
    mean = mean.sum((1, 3)) / count
    d = xg - mean[:, None, :, None]
    if carry:
        d = d * mask
    var = (d * d).sum((1, 3)) / count
    return mean, 1.0 / torch.sqrt(var + EPS)


def _act(z, act):
    if act == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    return z / (1 + torch.exp(-z)) if act == "silu" else z


def _gn_plain(s, dt):
    c = s["case"]
    x = s["x"].to(dt)
    xg = x.reshape(c["n"], -1, c["groups"], c["c"] // c["groups"])
    mean, rstd = _stats(xg, c["carry"])
    z = ((xg - mean[:, None, :, None]) * rstd[:, None, :, None]).reshape(
        x.shape) * s["gamma"].to(dt) + s["beta"].to(dt)
    if c["carry"]:
        z[..., -1] = x[..., -1]
    if s["residual"] is not None:
        z = z + s["residual"].to(dt)
    y = _act(z, c["act"])
    if c["carry"]:
        y[..., -1] = z[..., -1]
    return y, mean, rstd


def _gn_grad_plain(s, dt, mean, rstd):
    c = s["case"]
    x, gamma = s["x"].to(dt), s["gamma"].to(dt)
    shape = (c["n"], -1, c["groups"], c["c"] // c["groups"])
    xhat = ((x.reshape(shape) - mean[:, None, :, None])
            * rstd[:, None, :, None]).reshape(x.shape)
    dz = s["dy"].to(dt)
    if c["act"] != "none":
        z = xhat * gamma + s["beta"].to(dt)
        if s["residual"] is not None:
            z = z + s["residual"].to(dt)
        if c["act"] == "relu":
            d = (z > 0).to(dt)
        else:
            sig = 1 / (1 + torch.exp(-z))
            d = sig * (1 + z * (1 - sig))
        if c["carry"]:
            d[..., -1] = 1
        dz = dz * d
    own_dz = dz
    count = float(x[0].numel() // c["groups"])
    count = torch.full((c["groups"],), count, dtype=dt, device=x.device)
    if c["carry"]:
        own_dz = dz.clone()
        own_dz[..., -1] = 0
        count[-1] -= c["h"] * c["w"]
        count.clamp_(min=1)
    dgamma = (own_dz * xhat).sum((0, 1, 2))
    dbeta = own_dz.sum((0, 1, 2))
    dn = own_dz * gamma
    s1 = dn.reshape(shape).sum((1, 3)) / count
    s2 = (dn * xhat).reshape(shape).sum((1, 3)) / count
    dx = ((dn.reshape(shape) - s1[:, None, :, None]
           - xhat.reshape(shape) * s2[:, None, :, None])
          * rstd[:, None, :, None]).reshape(x.shape)
    if c["carry"]:
        dx[..., -1] = dz[..., -1]
    return dx, dz, dgamma, dbeta


def _mm_plain(s, dt):
    c = s["case"]
    a = s["a"].to(dt) * _spread(s["sa"].to(dt), c["m"], c["k"], 1)
    b = s["b"].to(dt) * _spread(s["sb"].to(dt), c["n"], c["k"], c["b_block"])
    y = a @ b.t()
    if s["bias"] is not None:
        y += s["bias"].to(dt)
    return _act(y, c["act"])


def _scores_plain(logits, targets, top_k):
    x = logits.float()
    rows, vocab = x.shape
    m = x.amax(1)
    empty = m == -math.inf
    m0 = torch.where(empty, torch.zeros_like(m), m)
    d = x - m0[:, None]
    e = torch.exp(d)
    s = e.sum(1)
    lse = m0 + torch.log(s)
    t = torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1)
    entropy = torch.where(empty, torch.zeros_like(s), torch.log(s) - t / s)
    given = targets >= 0
    at = targets.clamp(min=0).long()[:, None]
    xt = x.gather(1, at)
    lp = torch.where(empty, lse, xt[:, 0] - lse)
    ids = torch.arange(vocab, device=x.device)
    rank = ((x > xt) | ((x == xt) & (ids < at))).sum(1)
    out = {"lse": lse, "entropy": entropy,
           "logprob": torch.where(given, lp, torch.zeros_like(lp)),
           "rank": torch.where(given, rank, torch.full_like(rank, -1)).int()}
    if top_k:
        k = min(top_k, vocab)
        # ordered by value, then by the lower index: one whole number each
        bits = (x + 0.0).view(torch.int32)
        key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long()
        key = key * 2 ** 32 + (2 ** 32 - 1 - ids)
        top = 2 ** 32 - 1 - (torch.topk(key, k).values & (2 ** 32 - 1))
        v = x.gather(1, top)
        barred = v == -math.inf
        ids = torch.full((rows, top_k), -1, dtype=torch.int32,
                         device=x.device)
        lps = torch.full((rows, top_k), -math.inf, device=x.device)
        ids[:, :k] = torch.where(barred, torch.full_like(top, -1), top).int()
        lps[:, :k] = torch.where(barred, v, v - lse[:, None])
        out["top_ids"], out["top_logprobs"] = ids, lps
    return out


def _scores_grad(logits, s, dt, lse, entropy):
    x = logits.to(dt)
    g_lp, g_h = s["g_logprob"].to(dt), s["g_entropy"].to(dt)
    given = s["targets"] >= 0
    g_lp = torch.where(given, g_lp, torch.zeros_like(g_lp))
    empty = lse == -math.inf
    lse = torch.where(empty, torch.zeros_like(lse), lse)
    lp = x - lse[:, None]
    p = torch.exp(lp)
    h = torch.where(p > 0, lp, torch.zeros_like(lp)) + entropy[:, None]
    dx = p * (-g_lp[:, None] - g_h[:, None] * h)
    g_lp = torch.where(empty, torch.zeros_like(g_lp), g_lp)
    return dx.scatter_add_(1, s["targets"].clamp(min=0).long()[:, None],
                           g_lp[:, None])


# -------------------------------------------------------------------- runs

def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "group_norm":
        dt = DT[c["dtype"]]
        if not c["backward"]:
            y, mean, rstd = _gn_plain(s, torch.float32)
            return {"y": y.to(dt), "mean": mean, "rstd": rstd}
        dx, dr, dgamma, dbeta = _gn_grad_plain(s, torch.float32, s["mean"],
                                               s["rstd"])
        return {"dx": dx.to(dt), "dgamma": dgamma, "dbeta": dbeta,
                "dresidual": dr.to(dt) if c["residual"] else None}
    if c["op"] == "quantize":
        x = s["x"].t().contiguous() if c["transpose"] else s["x"]
        q, scales = _quantize(x, c["qtype"], c["block_rows"])
        return {"q": q, "scales": scales}
    if c["op"] == "matmul":
        return {"y": _mm_plain(s, torch.float32).to(DT[c["dtype"]])}
    if c["backward"]:
        return {"dlogits": _scores_grad(s["logits"], s, torch.float32,
                                        s["lse"], s["entropy"])
                .to(DT[c["dtype"]])}
    return _scores_plain(s["logits"], s["targets"], c["top_k"])


def _run_own(s):
    from paper_2609_16742_amd import ops
    c = s["case"]
    if c["op"] == "group_norm":
        kw = dict(gamma=s["gamma"], beta=s["beta"], residual=s["residual"],
                  act=c["act"], carry=c["carry"])
        if not c["backward"]:
            y, mean, rstd = ops.group_norm(s["x"], c["groups"], eps=EPS, **kw)
            return {"y": y, "mean": mean, "rstd": rstd}
        dx, dr, dgamma, dbeta = ops.group_norm_backward(
            s["dy"], s["x"], s["mean"], s["rstd"], c["groups"], **kw)
        return {"dx": dx, "dgamma": dgamma, "dbeta": dbeta, "dresidual": dr}
    if c["op"] == "quantize":
        q, scales = ops.fp8_quantize(s["x"], c["qtype"], c["block_rows"],
                                     transpose=c["transpose"])
        return {"q": q, "scales": scales}
    if c["op"] == "matmul":
        return {"y": ops.fp8_matmul(s["a"], s["sa"], s["b"], s["sb"],
                                    bias=s["bias"], act=c["act"],
                                    dtype=DT[c["dtype"]])}
    if c["backward"]:
        return {"dlogits": ops.token_scores_backward(
            s["logits"], s["targets"], s["lse"], s["entropy"],
            g_logprob=s["g_logprob"], g_entropy=s["g_entropy"])}
    r = ops.token_scores(s["logits"], s["targets"], c["top_k"])
    out = {"lse": r.lse, "entropy": r.entropy, "logprob": r.logprob,
           "rank": r.rank}
    if c["top_k"]:
        out["top_ids"], out["top_logprobs"] = r.top_ids, r.top_logprobs
    return out


# ---------------------------------------------------------- 64-bit results

def exact(case, seed):
    s = prepare(case, seed)
    return {"group_norm": _exact_gn, "quantize": _exact_quant,
            "matmul": _exact_mm, "scores": _exact_scores}[case["op"]](case, s)


def _exact_gn(c, s):
    """Image by image and group by group, from the definitions."""
    x, res = s["x"], s["residual"]
    gamma, beta = s["gamma"].double(), s["beta"].double()
    per = c["c"] // c["groups"]
    if c["backward"]:
        outs = {"dx": torch.empty(x.shape, dtype=torch.float64, device="cuda"),
                "dgamma": torch.zeros(c["c"], dtype=torch.float64,
                                      device="cuda"),
                "dbeta": torch.zeros(c["c"], dtype=torch.float64,
                                     device="cuda"),
                "dresidual": None}
        if res is not None:
            outs["dresidual"] = torch.empty_like(outs["dx"])
    else:
        outs = {"y": torch.empty(x.shape, dtype=torch.float64, device="cuda"),
                "mean": torch.zeros((c["n"], c["groups"]),
                                    dtype=torch.float64, device="cuda"),
                "rstd": torch.zeros((c["n"], c["groups"]),
                                    dtype=torch.float64, device="cuda")}
    for g in range(c["groups"]):
        lo, hi = g * per, (g + 1) * per
        ck = c["carry"] and hi == c["c"]
        ch = slice(lo, hi - 1 if ck else hi)
        if ck:
            z = x[..., -1].double()
            if c["backward"]:
                outs["dx"][..., -1] = s["dy"][..., -1].double()
                if res is not None:
                    outs["dresidual"][..., -1] = s["dy"][..., -1].double()
            else:
                outs["y"][..., -1] = z if res is None else \
                    z + res[..., -1].double()
        v = x[..., ch].double()
        if v.numel():
            var, mean = torch.var_mean(v, (1, 2, 3), correction=0,
                                       keepdim=True)
        else:
            mean = torch.zeros((c["n"], 1, 1, 1), dtype=torch.float64,
                               device="cuda")
            var = mean
        rstd = (var + EPS).rsqrt()
        xhat = (v - mean) * rstd
        z = xhat * gamma[ch] + beta[ch]
        if res is not None:
            z = z + res[..., ch].double()
        sig = torch.sigmoid(z)
        if not c["backward"]:
            outs["mean"][:, g], outs["rstd"][:, g] = mean.flatten(), \
                rstd.flatten()
            outs["y"][..., ch] = z if c["act"] == "none" else \
                z.clamp(min=0) if c["act"] == "relu" else z * sig
            continue
        dz = s["dy"][..., ch].double()
        if c["act"] == "relu":
            dz = dz * (z > 0)
        elif c["act"] == "silu":
            dz = dz * (sig + z * sig * (1 - sig))
        if res is not None:
            outs["dresidual"][..., ch] = dz
        outs["dbeta"][ch] = dz.sum((0, 1, 2))
        outs["dgamma"][ch] = (dz * xhat).sum((0, 1, 2))
        if v.numel():
            dn = dz * gamma[ch]
            dn = dn - dn.mean((1, 2, 3), keepdim=True) - xhat * (
                dn * xhat).mean((1, 2, 3), keepdim=True)
            outs["dx"][..., ch] = dn * rstd
    return outs


def _exact_quant(c, s):
    x = s["x"].double()
    if c["transpose"]:
        x = x.t()
    rows, cols = x.shape
    scales = torch.empty((_blocks(cols, BLOCK),
                          _blocks(rows, c["block_rows"])),
                         dtype=torch.float64, device="cuda")
    for i in range(scales.shape[0]):
        top = x[:, i * BLOCK:(i + 1) * BLOCK].abs().amax(1)
        if c["block_rows"] > 1:
            top = torch.stack([t.amax() for t in top.split(c["block_rows"])])
        scales[i] = top.clamp(min=2.0 ** -100) / F8_MAX[c["qtype"]]
    # which of two neighbours an 8-bit value is at a tie goes by the 32-bit
    # product that is rounded: no value of its own
    return {"q": None, "scales": scales}


def _exact_mm(c, s):
    y = torch.zeros((c["m"], c["n"]), dtype=torch.float64, device="cuda")
    for i in range(s["sa"].shape[0]):
        ks = slice(i * BLOCK, min((i + 1) * BLOCK, c["k"]))
        sb = s["sb"][i].double()
        if c["b_block"] > 1:
            sb = sb.repeat_interleave(c["b_block"])[:c["n"]]
        # products of 8-bit values and their sums over a block are exact
        y += (s["a"][:, ks].double() @ s["b"][:, ks].double().t()) \
            * s["sa"][i].double()[:, None] * sb
    if s["bias"] is not None:
        y += s["bias"].double()
    if c["act"] == "relu":
        y = y.clamp(min=0)
    elif c["act"] == "silu":
        y = y * torch.sigmoid(y)
    return {"y": y}


def _exact_scores(c, s):
    parts = []
    step = max(1, (1 << 27) // c["vocab"])
    for r in range(0, c["rows"], step):
        x = s["logits"][r:r + step].double()
        t = s["targets"][r:r + step].long()
        lse = torch.logsumexp(x, 1, keepdim=True)
        empty = lse == -math.inf
        lp = torch.where(empty, -math.inf, x - lse)
        p = torch.exp(lp)
        h = -torch.where(p > 0, p * lp, 0.0).sum(1, keepdim=True)
        if c["backward"]:
            glp = s["g_logprob"][r:r + step].double()[:, None]
            gh = s["g_entropy"][r:r + step].double()[:, None]
            dx = -gh * torch.where(p > 0, p * (lp + h), 0.0)
            one = torch.zeros_like(p)
            one.scatter_(1, t.clamp(min=0)[:, None], 1.0)
            dx += torch.where((t >= 0)[:, None] & ~empty, glp, 0.0) * (one - p)
            parts.append({"dlogits": dx})
            continue
        d = {"lse": lse[:, 0], "entropy": h[:, 0],
             "logprob": torch.where(t < 0, 0.0, lp.gather(
                 1, t.clamp(min=0)[:, None])[:, 0])}
        if c["top_k"]:
            k = min(c["top_k"], c["vocab"])
            d["top_logprobs"] = torch.full((x.shape[0], c["top_k"]),
                                           -math.inf, dtype=torch.float64,
                                           device="cuda")
            d["top_logprobs"][:, :k] = lp.sort(1, descending=True)[0][:, :k]
        parts.append(d)
    out = {k: torch.cat([d[k] for d in parts]) for k in parts[0]}
    if not c["backward"]:
        out["rank"] = None
        if c["top_k"]:
            out["top_ids"] = None
    return out
