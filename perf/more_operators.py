"""The operators of a head over a feature map's pixels, as timed cases.

Attention of queries over keys (maps' pixels as tokens, one pooling query over
many pixels, long causal sequences) and its backward pass, which recomputes the
probabilities; norms of queries and keys for each head with a rotation by
several position axes; the global norm of many gradients, and clipping.  Sizes
are those of the repository's networks (maps from 7x7 to 112x112, 512 channels,
parameters of its smallest and its largest network) and generic sizes of longer
sequences.

The plain forms compute in 32 bits with elementary torch operations (angles of
positions and sums over all gradients in 64).
"""

import math

import torch

own = False

DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6
BASE = 100.0
# What a plain pass holds of scores at a time, and the largest passes drawn:
# pairs of a query and a key (a gradient's count 2.5 times), elements of
# queries, keys and values, elements of a norm, of gradients.
HELD = 1 << 28
MOST_PAIRS = 2 * 16 * 8192 * 8192
MOST_TOKENS = 8 * 12544 * 2 * 8 * 128
MOST_NORM = 2 * 6272 * 40 * 128
MOST_GRADS = 138 * 10 ** 6


# ------------------------------------------------------------------- cases

def _attn(name, dtype, b, tq, tk, hq, hkv, d, causal=False, ragged=False,
          backward=False):
    return dict(name=name, op="attention", dtype=dtype, b=b, tq=tq, tk=tk,
                hq=hq, hkv=hkv, d=d, causal=causal, ragged=ragged,
                backward=backward)


def _turn(name, dtype, b, sizes, hq, hkv, d, interleaved=False, narrow="",
          backward=False):
    """`sizes`: extents of the position axes, as text ("8x28x28")."""
    return dict(name=name, op="norm_rotary", dtype=dtype, b=b, sizes=sizes,
                hq=hq, hkv=hkv, d=d, interleaved=interleaved, narrow=narrow,
                backward=backward)


def _clip(name, dtype, net, params, clipped=True):
    """Gradients of a network of `params` parameters: `net` is "thin" or
    "wide" (see _shapes)."""
    return dict(name=name, op="clip", dtype=dtype, net=net, params=params,
                clipped=clipped)


def listed():
    return [
        # One image's last map in a serving call, 8 heads of 64: latency.
        _attn("attn_f16_b1_7x7_h8x64", "f16", 1, 49, 49, 8, 8, 64),
        # Pooling, or one new token: a single query over up to 12544 keys of
        # 8 sequences of different lengths, 4 query heads to a key head.
        _attn("attn_bf16_b8_1q_12544_h32x128", "bf16", 8, 1, 12544, 32, 8,
              128, ragged=True),
        # A batch's 14x14 maps.
        _attn("attn_f16_b64_14x14_h8x64", "f16", 64, 196, 196, 8, 8, 64),
        # Long causal sequences, 8 query heads to a key head.
        _attn("attn_bf16_b2_8192_causal_h16x128", "bf16", 2, 8192, 8192, 16,
              2, 128, causal=True),
        # Training on a batch's last maps.
        _attn("attn_grad_f16_b64_7x7_h8x64", "f16", 64, 49, 49, 8, 8, 64,
              backward=True),
        # Training on large maps: 56x56 pixels.
        _attn("attn_grad_bf16_b2_56x56_h16x128", "bf16", 2, 3136, 3136, 16,
              16, 128, backward=True),
        # Odd lengths, an odd head size, causal, shared key heads.
        _attn("attn_grad_f16_b3_1025_causal_h12x80", "f16", 3, 1025, 1025,
              12, 4, 80, causal=True, ragged=True, backward=True),
        # Queries and keys of a batch's last maps, rows and columns.
        _turn("norm_rotary_f16_b64_7x7_h8x64", "f16", 64, "7x7", 8, 8, 64),
        # Queries and keys of clips of 8 frames.
        _turn("norm_rotary_bf16_b2_8x28x28_h32x128", "bf16", 2, "8x28x28", 32,
              8, 128),
        # The gradients of the same.
        _turn("norm_rotary_grad_bf16_b2_8x28x28_h32x128", "bf16", 2,
              "8x28x28", 32, 8, 128, backward=True),
        # The gradients of a small network: many short vectors.
        _clip("clip_f32_thin_270k", "f32", "thin", 270000),
        # The gradients of the largest network.
        _clip("clip_f32_wide_138m", "f32", "wide", MOST_GRADS),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice([_draw_attn, _draw_attn, _draw_attn, _draw_turn,
                           _draw_turn, _draw_clip])
        case = kind(rng)
        if _size(case) <= 1.0:
            del case["name"]
            return case


def _size(case):
    """The case's size against the largest of its kind."""
    c = case
    if c["op"] == "attention":
        pairs = c["b"] * c["hq"] * c["tq"] * c["tk"]
        return max((2.5 if c["backward"] else 1) * pairs / MOST_PAIRS,
                   c["b"] * (c["tq"] * c["hq"] + 2 * c["tk"] * c["hkv"])
                   * c["d"] / MOST_TOKENS)
    if c["op"] == "norm_rotary":
        return c["b"] * _pixels(c) * (c["hq"] + c["hkv"]) * c["d"] / MOST_NORM
    return c["params"] / MOST_GRADS


def _draw_attn(rng):
    hkv = rng.choice([1, 2, 3, 4, 8, 12, 16])
    hq = hkv * rng.choice([1, 1, 1, 2, 3, 4, 8])
    kind = rng.choice(["same", "same", "one", "cross"])
    tk = _log(rng, 1, 12544)
    tq = {"same": tk, "one": rng.choice([1, 1, 2, 4]),
          "cross": _log(rng, 1, 4096)}[kind]
    return _attn("", rng.choice(["f16", "bf16"]), _log(rng, 1, 64), tq, tk,
                 hq, hkv, rng.choice([32, 64, 64, 128, 128, 40, 72, 80, 96]),
                 causal=kind != "cross" and rng.random() < 0.4,
                 ragged=rng.random() < 0.4, backward=rng.random() < 0.5)


def _draw_turn(rng):
    axes = rng.choice([1, 2, 2, 3])
    side = _log(rng, 1, 112)
    sizes = {1: [_log(rng, 1, 8192)], 2: [side, max(1, side - rng.choice(
        [0, 0, 1, 3]))], 3: [rng.randint(1, 9), side, side]}[axes]
    hkv = rng.choice([1, 2, 4, 8, 16])
    dtype = rng.choice(["f32", "f16", "bf16"])
    return _turn("", dtype, _log(rng, 1, 64), "x".join(map(str, sizes)),
                 hkv * rng.choice([1, 1, 2, 4]), hkv,
                 rng.choice([32, 64, 128, 40, 80, 96]),
                 interleaved=rng.random() < 0.3,
                 narrow=rng.choice(["f16", "bf16"]) if dtype == "f32" else "",
                 backward=rng.random() < 0.5)


def _draw_clip(rng):
    return _clip("", rng.choice(["f32", "f32", "f16", "bf16"]),
                 rng.choice(["thin", "wide"]), _log(rng, 60000, MOST_GRADS),
                 clipped=rng.random() < 0.8)


def _pixels(c):
    n = 1
    for s in c["sizes"].split("x"):
        n *= int(s)
    return n


def _axes(c):
    """Pairs turned by each axis: the head's, shared out."""
    n, left = len(c["sizes"].split("x")), c["d"] // 2
    per = left // n // 4 * 4
    return tuple([left - per * (n - 1)] + [per] * (n - 1))


def _shapes(c):
    """Tensors of a network of so many parameters: 3x3 filters, each with
    three vectors, twice as wide every few layers; a wide one ends with three
    matrices that hold most."""
    shapes, left, width, layers = [], c["params"], 16, 6
    if c["net"] == "wide":
        side = int(math.sqrt(c["params"] * 0.89 / 7.25))
        shapes = [(side, 6 * side + side // 8), (side, side),
                  (side // 8, side)]
        left -= sum(a * b for a, b in shapes)
        width, layers = 32, 2
    while left > layers * (9 * width * width + 3 * width):
        for _ in range(layers):
            shapes += [(width, width, 3, 3), (width,), (width,), (width,)]
            left -= 9 * width * width + 3 * width
        width *= 2
    return shapes + [(max(1, left),)]


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    s = {"attention": _prepare_attn, "norm_rotary": _prepare_turn,
         "clip": _prepare_clip}[case["op"]](case, g)
    s["case"] = dict(case)
    return s


def _randn(g, *shape):
    return torch.randn(shape, device="cuda", generator=g)


def _lengths(g, b, t):
    """Between half of the longest and all of it; one sequence is full."""
    n = t - (torch.rand(b, device="cuda", generator=g) * (t // 2)).int()
    n[b // 2] = t
    return n.int()


def _prepare_attn(c, g):
    dt, b, d = DT[c["dtype"]], c["b"], c["d"]
    # queries and keys come of their norm, values are a part of the
    # projection's output
    s = {"q": _randn(g, b, c["tq"], c["hq"], d).to(dt),
         "k": _randn(g, b, c["tk"], c["hkv"], d).to(dt)}
    both = torch.empty((b, c["tk"], 2 * c["hkv"], d), dtype=dt, device="cuda")
    for i in range(b):
        both[i] = _randn(g, c["tk"], 2 * c["hkv"], d).to(dt)
    s["v"] = both[:, :, c["hkv"]:]
    s["k_lengths"] = s["q_lengths"] = None
    if c["ragged"]:
        s["k_lengths"] = _lengths(g, b, c["tk"])
        if c["tq"] == c["tk"]:
            s["q_lengths"] = s["k_lengths"]
    s["scale"] = d ** -0.5
    if c["backward"]:
        s["do"] = (_randn(g, b, c["tq"], c["hq"], d) / 64).to(dt)
        s["o"], s["lse"] = _attn_plain(s, c)
    return s


def _prepare_turn(c, g):
    dt, b, d, t = DT[c["dtype"]], c["b"], c["d"], _pixels(c)
    n = c["hq"] + c["hkv"]
    # queries and keys beside each other, as a projection writes them
    both = torch.empty((b, t, n, d), dtype=dt, device="cuda")
    for i in range(b):
        both[i] = (1.5 * _randn(g, t, n, d)).to(dt)
    sizes = [int(v) for v in c["sizes"].split("x")]
    grid = torch.meshgrid(*[torch.arange(v, dtype=torch.int32, device="cuda")
                            for v in sizes], indexing="ij")
    s = {"q": both[:, :, :c["hq"]], "k": both[:, :, c["hq"]:],
         "q_weight": 1 + 0.2 * _randn(g, d),
         "k_weight": 1 + 0.2 * _randn(g, d),
         "positions": torch.stack([v.flatten() for v in grid], 1).contiguous(),
         "axes": _axes(c)}
    s["frequencies"] = torch.cat([
        BASE ** (-torch.arange(p, device="cuda", dtype=torch.float32) / p)
        for p in s["axes"] if p])
    out = DT[c["narrow"]] if c["narrow"] else dt
    s["dtype"] = out
    if c["backward"]:
        s["dq"] = (_randn(g, b, t, c["hq"], d) / 64).to(out)
        s["dk"] = (_randn(g, b, t, c["hkv"], d) / 64).to(out)
    return s


def _prepare_clip(c, g):
    dt, shapes = DT[c["dtype"]], _shapes(c)
    grads = [(0.01 * _randn(g, *v)).to(dt) for v in shapes]
    norm = 0.01 * math.sqrt(c["params"])
    return {"grads": grads, "out": [torch.empty_like(v) for v in grads],
            "max_norm": norm * (0.25 if c["clipped"] else 4.0)}


# ------------------------------------------------------------- plain forms

def _hidden(s, c, i):
    """[tq, tk]: which pairs of sequence i take no part."""
    rows = torch.arange(c["tq"], device="cuda")[:, None]
    cols = torch.arange(c["tk"], device="cuda")[None]
    nq = c["tq"] if s["q_lengths"] is None else s["q_lengths"][i]
    nk = c["tk"] if s["k_lengths"] is None else s["k_lengths"][i]
    off = (rows >= nq) | (cols >= nk)
    if c["causal"]:
        off = off | (cols > rows + (nk - nq))
    return off


def _parts(c):
    """Parts of the batch whose scores are held at a time."""
    one = c["hq"] * c["tq"] * c["tk"]
    n = max(1, HELD // one)
    return [(i, min(c["b"], i + n)) for i in range(0, c["b"], n)]


def _probabilities(s, c, lo, hi, lse=None):
    """(q, k, v as [n, hkv, group * tq or tk, d], probabilities, lse)."""
    n, grp, d = hi - lo, c["hq"] // c["hkv"], c["d"]

    def rows(x):
        return x[lo:hi].float().view(n, c["tq"], c["hkv"], grp, d) \
            .permute(0, 2, 3, 1, 4).reshape(n, c["hkv"], grp * c["tq"], d)
    q = rows(s["q"])
    k = s["k"][lo:hi].float().permute(0, 2, 1, 3).contiguous()
    v = s["v"][lo:hi].float().permute(0, 2, 1, 3).contiguous()
    x = (q @ k.transpose(2, 3).contiguous()) * s["scale"]
    off = torch.stack([_hidden(s, c, i) for i in range(lo, hi)]) \
        if c["ragged"] else _hidden(s, c, 0)[None]
    x = x.view(n, c["hkv"], grp, c["tq"], c["tk"])
    x = x.masked_fill_(off[:, None, None], -math.inf).view(
        n, c["hkv"], grp * c["tq"], c["tk"])
    if lse is None:
        m = x.amax(3, keepdim=True)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        x = torch.exp(x.sub_(m))
        total = x.sum(3, keepdim=True)
        lse = m + torch.log(total)
        x = x / torch.where(total == 0, torch.ones_like(total), total)
    else:
        lse = lse[lo:hi].view(n, c["hkv"], grp * c["tq"], 1)
        x = torch.exp(x.sub_(torch.where(lse == -math.inf,
                                         torch.zeros_like(lse), lse)))
    return rows, q, k, v, x, lse


def _back(x, c, n):
    """[n, hkv, group * tq, d] as [n, tq, hq, d]."""
    grp = c["hq"] // c["hkv"]
    return x.view(n, c["hkv"], grp, c["tq"], -1).permute(0, 3, 1, 2, 4) \
        .reshape(n, c["tq"], c["hq"], -1)


def _attn_plain(s, c):
    dt = DT[c["dtype"]]
    o = torch.empty((c["b"], c["tq"], c["hq"], c["d"]), dtype=dt,
                    device="cuda")
    out_lse = torch.empty((c["b"], c["hq"], c["tq"]), device="cuda")
    for lo, hi in _parts(c):
        _, _, _, v, p, lse = _probabilities(s, c, lo, hi)
        o[lo:hi] = _back(p @ v, c, hi - lo).to(dt)
        out_lse[lo:hi] = lse.view(hi - lo, c["hq"], c["tq"])
    return o, out_lse


def _attn_grad_plain(s, c):
    dt = DT[c["dtype"]]
    dq = torch.empty(s["q"].shape, dtype=dt, device="cuda")
    dk = torch.empty(s["k"].shape, dtype=dt, device="cuda")
    dv = torch.empty(s["k"].shape, dtype=dt, device="cuda")
    for lo, hi in _parts(c):
        rows, q, k, v, p, _ = _probabilities(s, c, lo, hi, s["lse"])
        do, o = rows(s["do"]), rows(s["o"])
        delta = (do * o).sum(3, keepdim=True)
        dv[lo:hi] = (p.transpose(2, 3).contiguous() @ do).permute(
            0, 2, 1, 3).to(dt)
        ds = (do @ v.transpose(2, 3).contiguous()).sub_(delta).mul_(p)
        ds *= s["scale"]
        dq[lo:hi] = _back(ds @ k, c, hi - lo).to(dt)
        dk[lo:hi] = (ds.transpose(2, 3).contiguous() @ q).permute(
            0, 2, 1, 3).to(dt)
    return dq, dk, dv


def _angles(s):
    """[t, pairs] in 64 bits."""
    axis = torch.repeat_interleave(
        torch.arange(len(s["axes"]), device="cuda"),
        torch.tensor(s["axes"], device="cuda"))
    return s["positions"].double()[:, axis] * s["frequencies"].double()


def _halves(x, c):
    if c["interleaved"]:
        return x[..., 0::2], x[..., 1::2]
    return x[..., :c["d"] // 2], x[..., c["d"] // 2:]


def _join(a, b, c):
    if c["interleaved"]:
        return torch.stack([a, b], -1).flatten(-2)
    return torch.cat([a, b], -1)


def _turn_plain(x, w, cos, sin, c, dt):
    x = x.float()
    z = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w
    a, b = _halves(z, c)
    return _join(a * cos - b * sin, a * sin + b * cos, c).to(dt)


def _turn_grad_plain(dy, x, w, cos, sin, c):
    dt, x, dy = x.dtype, x.float(), dy.float()
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    xhat = x * rstd
    a, b = _halves(dy, c)
    dz = _join(a * cos + b * sin, b * cos - a * sin, c)
    dw = (dz * xhat).sum((0, 1, 2))
    dn = dz * w
    dx = (dn - xhat * (dn * xhat).mean(-1, keepdim=True)) * rstd
    return dx.to(dt), dw


# -------------------------------------------------------------------- runs

def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "attention":
        if c["backward"]:
            dq, dk, dv = _attn_grad_plain(s, c)
            return {"dq": dq, "dk": dk, "dv": dv}
        o, lse = _attn_plain(s, c)
        return {"o": o, "lse": lse}
    if c["op"] == "norm_rotary":
        a = _angles(s)
        cos = torch.cos(a).float()[:, None]
        sin = torch.sin(a).float()[:, None]
        if c["backward"]:
            dq, dqw = _turn_grad_plain(s["dq"], s["q"], s["q_weight"], cos,
                                       sin, c)
            dk, dkw = _turn_grad_plain(s["dk"], s["k"], s["k_weight"], cos,
                                       sin, c)
            return {"dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw}
        return {"q": _turn_plain(s["q"], s["q_weight"], cos, sin, c,
                                 s["dtype"]),
                "k": _turn_plain(s["k"], s["k_weight"], cos, sin, c,
                                 s["dtype"])}
    squares = [(g.double() ** 2).sum() for g in s["grads"]]
    norm = torch.sqrt(torch.stack(squares).sum())
    factor = torch.clamp(s["max_norm"] / norm, max=1.0).float()
    for g, o in zip(s["grads"], s["out"]):
        o.copy_(g.float() * factor)
    return {"out": s["out"], "norm": norm.float()}


def _run_own(s):
    from paper_2609_16742_amd import ops
    c = s["case"]
    if c["op"] == "attention":
        kw = dict(causal=c["causal"], q_lengths=s["q_lengths"],
                  k_lengths=s["k_lengths"], scale=s["scale"])
        if c["backward"]:
            dq, dk, dv = ops.attention_backward(
                s["do"], s["q"], s["k"], s["v"], s["o"], s["lse"], **kw)
            return {"dq": dq, "dk": dk, "dv": dv}
        o, lse = ops.attention(s["q"], s["k"], s["v"], **kw)
        return {"o": o, "lse": lse}
    if c["op"] == "norm_rotary":
        kw = dict(q_weight=s["q_weight"], k_weight=s["k_weight"],
                  positions=s["positions"], frequencies=s["frequencies"],
                  axes=s["axes"], interleaved=c["interleaved"], eps=EPS)
        if c["backward"]:
            dq, dk, dqw, dkw = ops.head_norm_rotary_backward(
                s["dq"], s["dk"], s["q"], s["k"], **kw)
            return {"dq": dq, "dk": dk, "dq_weight": dqw, "dk_weight": dkw}
        q, k = ops.head_norm_rotary(s["q"], s["k"], dtype=s["dtype"], **kw)
        return {"q": q, "k": k}
    out, norm = ops.clip_gradients(s["grads"], s["max_norm"], out=s["out"])
    return {"out": out, "norm": norm}


# ---------------------------------------------------------- 64-bit results

def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attn, "norm_rotary": _exact_turn,
            "clip": _exact_clip}[case["op"]](case, s)


def _exact_attn(c, s):
    """Head by head, and so many rows at a time, from the definitions."""
    f8 = dict(dtype=torch.float64, device="cuda")
    shape = (c["b"], c["tq"], c["hq"], c["d"])
    if c["backward"]:
        out = {"dq": torch.zeros(shape, **f8),
               "dk": torch.zeros(s["k"].shape, **f8),
               "dv": torch.zeros(s["k"].shape, **f8)}
    else:
        out = {"o": torch.zeros(shape, **f8),
               "lse": torch.full((c["b"], c["hq"], c["tq"]), -math.inf, **f8)}
    if c["b"] * c["hq"] * (1 + c["tq"] * c["tk"] / 2 ** 26) > 4096:
        return None
    nq = [c["tq"]] * c["b"] if s["q_lengths"] is None \
        else s["q_lengths"].tolist()
    nk = [c["tk"]] * c["b"] if s["k_lengths"] is None \
        else s["k_lengths"].tolist()
    step = max(1, (1 << 27) // c["tk"])
    for i in range(c["b"]):
        for h in range(c["hq"]):
            kh = h // (c["hq"] // c["hkv"])
            k, v = s["k"][i, :nk[i], kh].double(), s["v"][i, :nk[i], kh].double()
            for r in range(0, nq[i], step):
                e = min(r + step, nq[i])
                q = s["q"][i, r:e, h].double()
                x = torch.mm(q, k.t()) * s["scale"]
                if c["causal"]:
                    last = torch.arange(r, e, device="cuda") + nk[i] - nq[i]
                    x[torch.arange(nk[i], device="cuda")[None]
                      > last[:, None]] = -math.inf
                lse = torch.logsumexp(x, 1, keepdim=True)
                p = torch.where(lse == -math.inf, 0.0, torch.exp(x - lse))
                o = torch.mm(p, v)
                if not c["backward"]:
                    out["o"][i, r:e, h], out["lse"][i, h, r:e] = o, lse[:, 0]
                    continue
                do = s["do"][i, r:e, h].double()
                ds = p * (torch.mm(do, v.t()) - (do * o).sum(1, keepdim=True))
                ds *= s["scale"]
                out["dv"][i, :nk[i], kh] += torch.mm(p.t(), do)
                out["dk"][i, :nk[i], kh] += torch.mm(ds.t(), q)
                out["dq"][i, r:e, h] = torch.mm(ds, k)
    return out


def _exact_turn(c, s):
    """Pairs as complex numbers."""
    t = _pixels(c)
    turn = torch.empty((t, c["d"] // 2), dtype=torch.complex128, device="cuda")
    at = 0
    for a, n in enumerate(s["axes"]):
        angle = torch.outer(s["positions"][:, a].double(),
                            s["frequencies"][at:at + n].double())
        turn[:, at:at + n] = torch.polar(torch.ones_like(angle), angle)
        at += n

    def pairs(x):
        x = x.double()
        if c["interleaved"]:
            x = x.unflatten(-1, (-1, 2))
            return torch.complex(x[..., 0].contiguous(), x[..., 1].contiguous())
        lo, hi = x.chunk(2, -1)
        return torch.complex(lo.contiguous(), hi.contiguous())

    def flat(z):
        if c["interleaved"]:
            return torch.view_as_real(z).flatten(-2)
        return torch.cat([z.real, z.imag], -1)

    out = {}
    for n in "qk":
        x, w = s[n].double(), s[n + "_weight"].double()
        size = torch.sqrt(x.pow(2).mean(-1, keepdim=True) + EPS)
        if not c["backward"]:
            out[n] = flat(pairs(x / size * w) * turn[:, None])
            continue
        dz = flat(pairs(s["d" + n]) * turn.conj()[:, None])
        out["d%s_weight" % n] = (dz * x / size).sum((0, 1, 2))
        dz = dz * w
        out["d" + n] = dz / size - x * (dz * x).mean(-1, keepdim=True) / size ** 3
    if c["backward"]:
        return {k: out[k] for k in ("dq", "dk", "dq_weight", "dk_weight")}
    return out


def _exact_clip(c, s):
    total = sum(float(torch.linalg.vector_norm(g.double())) ** 2
                for g in s["grads"])
    norm = math.sqrt(total)
    factor = s["max_norm"] / norm if norm > s["max_norm"] else 1.0
    return {"out": [g.double() * factor for g in s["grads"]],
            "norm": torch.tensor(norm, dtype=torch.float64, device="cuda")}


# -------------------------------------------------------------------- work

def work(case):
    c = case
    if c["op"] == "attention":
        # (lengths of ragged sequences: three quarters of the longest)
        tq, tk = float(c["tq"]), float(c["tk"])
        if c["ragged"]:
            part = (1 + 0.75 * (c["b"] - 1)) / c["b"]
            tk *= part
            if c["tq"] == c["tk"]:
                tq *= part
        pairs = c["b"] * c["hq"] * tq * tk
        if c["causal"]:
            short = min(tq, tk)
            pairs -= c["b"] * c["hq"] * short * (short - 1) / 2
        rows, keys = c["b"] * tq * c["hq"], c["b"] * tk * c["hkv"]
        if c["backward"]:
            return {"bytes": (rows * 4 + keys * 4) * c["d"] * 2 + rows * 4,
                    "flops": 10.0 * c["d"] * pairs}
        return {"bytes": (rows * 2 + keys * 2) * c["d"] * 2 + rows * 4,
                "flops": 4.0 * c["d"] * pairs}
    if c["op"] == "norm_rotary":
        e = c["b"] * _pixels(c) * (c["hq"] + c["hkv"]) * c["d"]
        i = torch.empty(0, dtype=DT[c["dtype"]]).element_size()
        o = torch.empty(0, dtype=DT[c["narrow"] or c["dtype"]]).element_size()
        if c["backward"]:
            return {"bytes": float(e * (2 * i + o)), "flops": 16.0 * e}
        return {"bytes": float(e * (i + o)), "flops": 8.0 * e}
    i = torch.empty(0, dtype=DT[c["dtype"]]).element_size()
    e = sum(math.prod(v) for v in _shapes(c))
    return {"bytes": 2.0 * e * i, "flops": 3.0 * e}
