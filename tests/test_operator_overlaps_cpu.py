"""Outputs of attention and head norms that lie over inputs or over each other:
refused by the C entry points before anything is enqueued, so no GPU is needed.
What is accepted reaches the launch, which a machine without a GPU reports as an
error of the device."""

import ctypes
import itertools
import random

import pytest

ctc = pytest.importorskip("paper_2609_16742_amd.ctc")

A = 1 << 40                       # addresses far apart, that nothing reads
FAR = 1 << 30
ARG = ctc.CTC_ERR_ARG


def heads(at, *strides):
    return ctc.ctc_heads(at, (ctypes.c_int64 * 3)(*strides))


def status(f, *args):
    try:
        f(*args)
    except ctc.CtcError as e:
        return e.status, str(e)
    return 0, ""


def refused(f, *args):
    s, text = status(f, *args)
    return s == ARG and "overlap" in text


@pytest.fixture(autouse=True)
def no_gpu():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the accepted calls would run on their made-up addresses")


def attention(b=2, tq=100, tk=100, hq=4, hk=4, d=64):
    return ctc.ctc_attention(ctc.CTC_F16, b, tq, tk, hq, hk, d, 0, 0.125, None, None)


def forward(a, q, k, v, o, lse=A + 9 * FAR):
    ctc.ctc_attention_forward(a, q, k, v, o, lse, A + 10 * FAR, 1 << 29, None)


def backward(a, do, q, k, v, o, dq, dk, dv, lse=A + 9 * FAR):
    ctc.ctc_attention_backward(a, do, q, k, v, o, lse, dq, dk, dv,
                               A + 10 * FAR, 1 << 29, None)


def plain(i, h=4, d=64, t=100, shift=0):
    return heads(A + i * FAR + shift, t * h * d, h * d, d)


def test_forward():
    a = attention()
    q, k, v, o = (plain(i) for i in range(4))
    assert not refused(forward, a, q, k, v, o)
    assert not refused(forward, a, q, k, v, q)              # in place
    for bad in (k, v, plain(0, shift=128), plain(1, shift=2 * 100 * 256 * 2 - 16),
                plain(0, shift=2 * 64), plain(1, shift=-2 * 100 * 256 * 2 + 16)):
        assert refused(forward, a, q, k, v, bad)
    # behind the last value, and in front of the first
    for fine in (plain(1, shift=2 * 100 * 256 * 2), plain(1, shift=-2 * 100 * 256 * 2)):
        assert not refused(forward, a, q, k, v, fine)
    # the queries in another order
    assert refused(forward, a, q, k, v, heads(A, 100 * 256, 64, 6400))
    # queries that are the keys too
    assert refused(forward, a, q, q, v, q)
    for at in (A, A + FAR + 64, A + 3 * FAR + 32, A + 2 * FAR - 4):
        assert refused(forward, a, q, k, v, o, at)


def test_backward():
    a = attention()
    do, q, k, v, o, dq, dk, dv = (plain(i) for i in range(8))
    fine = dict(do=do, q=q, k=k, v=v, o=o, dq=dq, dk=dk, dv=dv)

    def call(**change):
        return refused(lambda: backward(a, **{**fine, **change}))
    assert not call()
    # keys' and values' gradients in place
    for change in (dict(dk=k), dict(dv=v), dict(dk=k, dv=v), dict(dk=v, dv=k), dict(dv=k),
                   dict(k=k, v=k, dk=k), dict(k=k, v=k, dv=k)):
        assert not call(**change)
    for change in (dict(dk=dv), dict(dq=dk), dict(dq=dv), dict(k=k, v=k, dk=k, dv=k),
                   dict(dq=q), dict(dq=do), dict(dq=o), dict(dq=k), dict(dq=v),
                   dict(dk=q), dict(dk=do), dict(dk=o), dict(dv=q), dict(dv=do), dict(dv=o),
                   dict(dk=plain(2, shift=128)), dict(dv=plain(2, shift=256)),
                   dict(dk=heads(A + 2 * FAR, 100 * 256, 64, 6400)),
                   dict(lse=A + 5 * FAR + 16), dict(lse=A + 6 * FAR)):
        assert call(**change), change


def test_parts_of_one_buffer():
    """Queries, keys and values side by side in a projection, their gradients
    in another, heads that share keys, lengths that differ."""
    for b, tq, tk, hq, hk, d, pad in itertools.product(
            (1, 3), (1, 70), (1, 100), (4, 8), (1, 2), (8, 64), (0, 8)):
        a = attention(b, tq, tk, hq, hk, d)
        row = (hq + 2 * hk) * (d + pad) + 16
        step = max(tq, tk) * row

        def part(at, first):
            return heads(A + at * FAR + 2 * first * (d + pad), step, row, d + pad)
        q, k, v = part(0, 0), part(0, hq), part(0, hq + hk)
        dq, dk, dv = part(1, 0), part(1, hq), part(1, hq + hk)
        do, o = plain(3, hq, d, tq), plain(4, hq, d, tq)
        assert not refused(backward, a, do, q, k, v, o, dq, dk, dv)
        assert not refused(backward, a, do, q, k, v, o, dq, k, v)
        assert not refused(forward, a, q, k, v, o)
        if hk > 1:
            # one head further: the values' first is the keys' last
            assert refused(backward, a, do, q, k, v, o, dq, dk, part(1, hq + hk - 1))


def test_against_all_elements():
    """Small tensors with strides of all kinds, told apart as their elements
    are."""
    rng = random.Random(3)
    seen = {False: 0, True: 0}
    for _ in range(3000):
        b, t, h, d = rng.choice([1, 2]), rng.randint(1, 4), rng.randint(1, 3), 8
        a = attention(b, t, t, h, h, d)

        def strides():
            order = [0, 1, 2]
            rng.shuffle(order)
            size, s, span = (b, t, h), [0, 0, 0], d
            for i in order:
                s[i] = span + 8 * rng.choice([0, 0, 1, 3, 6])
                span = s[i] * size[i]
            return s

        def elements(at, s):
            return {at + 2 * (i * s[0] + j * s[1] + x * s[2] + e) for i in range(b)
                    for j in range(t) for x in range(h) for e in range(d)}
        ks, os = strides(), strides()
        shift = 16 * rng.randint(-60, 60)
        want = bool(elements(0, ks) & elements(shift, os))
        k, o = heads(A + FAR, *ks), heads(A + FAR + shift, *os)
        got = refused(forward, a, plain(0), k, plain(2), o)
        assert got == want, (b, t, h, ks, os, shift)
        seen[want] += 1
    assert min(seen.values()) > 300


def rotary(dtype=ctc.CTC_F16, ytype=ctc.CTC_F16, b=2, t=49, hq=4, hk=4, d=64):
    return ctc.ctc_head_rotary(dtype, ytype, b, t, hq, hk, d, 1, 1e-6, A + 8 * FAR,
                               A + 8 * FAR + 4096, 0, 0, (ctypes.c_int32 * 4)(), 0, None, None)


def norm_forward(h, q, k, yq, yk):
    ctc.ctc_head_norm_rotary_forward(h, q, k, yq, yk, None)


def norm_backward(h, dyq, dyk, q, k, dq, dk, dqw=A + 9 * FAR, dkw=A + 9 * FAR + 256):
    ctc.ctc_head_norm_rotary_backward(h, dyq, dyk, q, k, dq, dk, dqw, dkw, A + 10 * FAR,
                                      1 << 29, None)


def test_head_norms():
    h = rotary()
    q, k, x, y, u, v = (plain(i, t=49) for i in range(6))
    assert not refused(norm_forward, h, q, k, x, y)
    assert not refused(norm_forward, h, q, k, q, k)
    assert not refused(norm_forward, h, q, q, x, y)
    for bad in ((k, y), (x, q), (k, q), (x, x), (plain(0, t=49, shift=128), y), (q, q),
                (x, heads(A + 8 * FAR - 128, 49 * 256, 256, 64))):
        assert refused(norm_forward, h, q, k, *bad)
    assert refused(norm_forward, h, q, q, q, y)             # the other reads it
    # in place, but of another type
    narrow = rotary(ctc.CTC_F32, ctc.CTC_F16)
    assert refused(norm_forward, narrow, q, k, q, y)
    assert not refused(norm_forward, narrow, q, k, x, y)
    assert not refused(norm_backward, h, x, y, q, k, u, v)
    for fine in ((x, y), (q, k), (x, k), (q, y)):
        assert not refused(norm_backward, h, x, y, q, k, *fine)
    for bad in ((y, v), (k, v), (u, x), (u, q), (u, u), (plain(2, t=49, shift=64), v)):
        assert refused(norm_backward, h, x, y, q, k, *bad)
    assert refused(norm_backward, narrow, x, y, q, k, x, v)
    for bad in (dict(dqw=A + 9 * FAR + 128), dict(dkw=A + 4 * FAR + 64), dict(dqw=A + 2 * FAR),
                dict(dqw=A + 8 * FAR), dict(dkw=A)):
        assert refused(lambda: norm_backward(h, x, y, q, k, u, v, **bad)), bad
    # queries and keys of one projection, their gradients over each other's
    # buffer in place, one without keys
    t, row = 49, 64 * 12
    part = [heads(A + 2 * i * 256, t * row, row, 64) for i in range(2)]
    grad = [heads(A + FAR + 2 * i * 256, t * row, row, 64) for i in range(2)]
    assert not refused(norm_forward, h, *part, *part)
    assert not refused(norm_forward, h, *part, *grad)
    assert not refused(norm_backward, h, *grad, *part, *grad)
    assert refused(norm_backward, h, *grad, *part, grad[1], grad[0])
    alone = rotary(hk=0)
    none = heads(0, 0, 0, 0)
    assert not refused(norm_forward, alone, q, none, q, none)
    assert not refused(norm_backward, alone, x, none, q, none, x, none, A + 9 * FAR, None)


def test_clipping_norm():
    """The norm over a gradient or over what one becomes."""
    def call(norm, *g):
        grads = (ctc.ctc_gradient * len(g))(*[ctc.ctc_gradient(*v, 0) for v in g])
        ctc.ctc_clip_gradients(len(g), grads, 1.0, norm, A + 10 * FAR, 1 << 29, None)
    x, y = A, A + FAR
    for g in (((x, y, 100, ctc.CTC_F32),), ((x, x, 100, ctc.CTC_F32),),
              ((x, x, 200, ctc.CTC_F16), (y, y, 200, ctc.CTC_BF16))):
        for at in (x, x + 396, x + 399, x - 3):
            assert refused(call, at, *g)
        for at in (x - 4, x + 400, y + 400, A + 2 * FAR, None):
            assert not refused(call, at, *g)
    for at in (y, y + 396):
        assert refused(call, at, (x, y, 100, ctc.CTC_F32))
