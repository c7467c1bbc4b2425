"""Refusals of the C entry points of attention, head norms and clipping:
everything is checked before anything is enqueued, so no GPU is needed."""

import ctypes

import pytest

ctc = pytest.importorskip("paper_2609_16742_amd.ctc")

P = 1 << 20                      # an address that no refused call reads
F32, F16, BF16, E4M3 = ctc.CTC_F32, ctc.CTC_F16, ctc.CTC_BF16, ctc.CTC_E4M3
ARG, UNSUPPORTED, WORKSPACE = (ctc.CTC_ERR_ARG, ctc.CTC_ERR_UNSUPPORTED,
                               ctc.CTC_ERR_WORKSPACE)
NAN, INF = float("nan"), float("inf")


def heads(at=P, *strides):
    return ctc.ctc_heads(at, (ctypes.c_int64 * 3)(*strides))


def _refused(status, f, *args):
    with pytest.raises(ctc.CtcError) as e:
        f(*args)
    assert e.value.status == status, str(e.value)


def _attention(**change):
    a = dict(dtype=F16, batch=2, queries=100, keys=300, q_heads=8, k_heads=2,
             head=64, causal=0, scale=0.125, q_lengths=None, k_lengths=None)
    assert set(change) <= set(a)
    a.update(change)
    return ctc.ctc_attention(*a.values())


Q = heads(P, 51200, 512, 64)
K = heads(P, 38400, 128, 64)


def _forward(a, q=Q, k=K, v=K, o=Q, lse=P, ws=P, ws_bytes=1 << 30):
    ctc.ctc_attention_forward(a, q, k, v, o, lse, ws, ws_bytes, None)


def _backward(a, do=Q, q=Q, k=K, v=K, o=Q, lse=P, dq=Q, dk=K, dv=K, ws=P,
              ws_bytes=1 << 30):
    ctc.ctc_attention_backward(a, do, q, k, v, o, lse, dq, dk, dv, ws,
                               ws_bytes, None)


@pytest.mark.parametrize("call", [_forward, _backward])
@pytest.mark.parametrize("status,change", [
    (ARG, dict(dtype=F32)), (ARG, dict(dtype=E4M3)), (ARG, dict(batch=-1)),
    (ARG, dict(queries=-1)), (ARG, dict(keys=-1)), (ARG, dict(q_heads=0)),
    (ARG, dict(k_heads=0)), (ARG, dict(k_heads=3)), (ARG, dict(head=0)),
    (ARG, dict(head=60)), (ARG, dict(head=136)), (ARG, dict(scale=0.0)),
    (ARG, dict(scale=-1.0)), (ARG, dict(scale=1e-35)), (ARG, dict(scale=NAN)), (ARG, dict(scale=INF)),
    (UNSUPPORTED, dict(keys=(1 << 30) + 1)),
    (UNSUPPORTED, dict(queries=1 << 29)),
    (UNSUPPORTED, dict(q_heads=1 << 18)),
    (UNSUPPORTED, dict(batch=1 << 22))], ids=str)
def test_attention_sizes(call, status, change):
    _refused(status, call, _attention(**change))


def test_attention_tensors():
    a = _attention()
    bad = [(ARG, None), (ARG, heads(0, 51200, 512, 64)),
           (ARG, heads(P + 8, 51200, 512, 64)), (ARG, heads(P, 51200, 512, 60)),
           (ARG, heads(P, 51200, 516, 64)), (ARG, heads(P, 51201, 512, 64)),
           (ARG, heads(P, 51200, -512, 64)),
           (UNSUPPORTED, heads(P, 51200, 1 << 23, 64)),
           (UNSUPPORTED, heads(P, 51200, 512, 1 << 28))]
    for status, h in bad:
        for n in ("q", "o"):
            _refused(status, lambda: _forward(a, **{n: h}))
        for n in ("do", "q", "o", "dq"):
            _refused(status, lambda: _backward(a, **{n: h}))
    for n in ("k", "v"):
        _refused(ARG, lambda: _forward(a, **{n: None}))
        _refused(UNSUPPORTED, lambda: _forward(a, **{n: heads(P, 8, 1 << 23, 64)}))
    # outputs that overlap themselves (inputs may: a broadcast gradient)
    for h in (heads(P, 51200, 0, 64), heads(P, 51200, 512, 56), heads(P, 8, 512, 64),
              heads(P, 51200, 256, 64), heads(P, 25600, 512, 64)):
        _refused(ARG, lambda: _forward(a, o=h))
        _refused(ARG, lambda: _backward(a, dq=h))
        _refused(ARG, lambda: _backward(a, dk=heads(P, 0, 128, 64)))
    _refused(ARG, lambda: _forward(a, lse=None))
    _refused(ARG, lambda: _backward(a, lse=None))


def test_attention_workspaces():
    few = _attention(queries=1, keys=100000)
    need = ctc.ctc_attention_workspace_bytes(few, 0)
    assert need > 0 and ctc.ctc_attention_workspace_bytes(_attention(batch=512), 0) == 0
    for ws, n in ((None, need), (P, need - 1), (P, 0)):
        _refused(WORKSPACE, lambda: _forward(few, ws=ws, ws_bytes=n))
    _refused(ARG, lambda: _forward(few, ws=P + 4, ws_bytes=need))
    need = ctc.ctc_attention_workspace_bytes(few, 1)
    far = heads(P, 12800000, 128, 64)
    _refused(WORKSPACE, lambda: _backward(few, dk=far, dv=far, ws_bytes=need - 1))
    # up to 64 rows and keys need none
    assert ctc.ctc_attention_workspace_bytes(
        _attention(queries=16, keys=64), 1) == 0
    assert ctc.ctc_attention_workspace_bytes(_attention(queries=17, keys=64), 1) > 0


def test_sizes_of_nothing():
    """Valid calls that do nothing: no pointer is read."""
    none = heads(0, 0, 0, 0)
    for a in (_attention(batch=0), _attention(queries=0)):
        ctc.ctc_attention_forward(a, none, none, none, none, None, None, 0, None)
    for a in (_attention(batch=0), _attention(queries=0, keys=0)):
        ctc.ctc_attention_backward(a, none, none, none, none, none, None, none,
                                   none, none, None, 0, None)
    h = _rotary(batch=0)
    ctc.ctc_head_norm_rotary_forward(h, none, none, none, none, None)
    ctc.ctc_clip_gradients(0, None, 1.0, None, None, 0, None)


def _rotary(pairs=(16, 16, 0, 0), **change):
    a = dict(dtype=F16, ytype=F16, batch=2, tokens=49, q_heads=8, k_heads=8,
             head=64, norm=1, eps=1e-6, q_weight=P, k_weight=P, interleaved=0,
             axes=2, pairs=(ctypes.c_int32 * 4)(*pairs), per_image=0,
             positions=P, frequencies=P)
    assert set(change) <= set(a)
    a.update(change)
    return ctc.ctc_head_rotary(*a.values())


H = heads(P, 49 * 512, 512, 64)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(dtype=E4M3)), (ARG, dict(ytype=F32)), (ARG, dict(ytype=BF16)),
    (ARG, dict(batch=-1)), (ARG, dict(tokens=-1)), (ARG, dict(q_heads=0)),
    (ARG, dict(k_heads=-1)), (ARG, dict(head=63)), (ARG, dict(head=514)),
    (ARG, dict(eps=-1.0)), (ARG, dict(eps=NAN)), (ARG, dict(axes=5)),
    (ARG, dict(axes=-1)), (ARG, dict(pairs=(17, 16, 0, 0))),
    (ARG, dict(pairs=(-1, 4, 0, 0))), (ARG, dict(positions=None)),
    (ARG, dict(frequencies=None)),
    (UNSUPPORTED, dict(head=258, pairs=(64, 64, 0, 0))),
    (UNSUPPORTED, dict(head=130, pairs=(1, 0, 0, 0))),
    (UNSUPPORTED, dict(batch=1 << 20, tokens=1 << 20))], ids=str)
def test_head_norm_sizes(status, change):
    h = _rotary(**change)
    _refused(status, lambda: ctc.ctc_head_norm_rotary_forward(h, H, H, H, H, None))
    _refused(status, lambda: ctc.ctc_head_norm_rotary_backward(
        h, H, H, H, H, H, H, P, P, P, 1 << 30, None))


def test_head_norm_tensors():
    h = _rotary()
    twice = heads(P, 49 * 512, 256, 64)
    for i in range(4):
        t = [H] * 4
        t[i] = None
        _refused(ARG, lambda: ctc.ctc_head_norm_rotary_forward(h, *t, None))
        if i > 1:
            t[i] = twice
            _refused(ARG, lambda: ctc.ctc_head_norm_rotary_forward(h, *t, None))
    for i in range(6):
        t = [H] * 6
        t[i] = None
        _refused(ARG, lambda: ctc.ctc_head_norm_rotary_backward(
            h, *t, P, P, P, 1 << 30, None))
    need = ctc.ctc_head_norm_rotary_workspace_bytes(h)
    _refused(WORKSPACE, lambda: ctc.ctc_head_norm_rotary_backward(
        h, *[H] * 6, P, P, P, need - 1, None))
    # (up to 128 values any number of pairs, more by twos and fours)
    for head, pairs in ((126, 63), (128, 1), (256, 2), (512, 4), (6, 3)):
        ctc.ctc_head_norm_rotary_workspace_bytes(_rotary(head=head, pairs=(pairs, 0, 0, 0)))


def _gradients(*g):
    return (ctc.ctc_gradient * len(g))(*[ctc.ctc_gradient(*v, 0) for v in g])


def _clip(*g, max_norm=1.0, ws=P, ws_bytes=1 << 30):
    ctc.ctc_clip_gradients(len(g), _gradients(*g), max_norm, P, ws, ws_bytes, None)


def test_clipping():
    A, B = 1 << 30, 1 << 31
    _refused(ARG, lambda: _clip((A, B, 10, E4M3)))
    _refused(ARG, lambda: _clip((A, B, -1, F32)))
    _refused(ARG, lambda: _clip((None, B, 10, F32)))
    _refused(ARG, lambda: _clip((A, None, 10, F32)))
    for n in (-1.0, NAN, -INF):
        _refused(ARG, lambda: _clip((A, B, 10, F32), max_norm=n))
    _refused(UNSUPPORTED, lambda: _clip((A, B, 1 << 44, F32)))
    # outputs over each other, over another's values, over their own in part
    _refused(ARG, lambda: _clip((A, B, 10, F32), (A + 64, B + 36, 10, F32)))
    _refused(ARG, lambda: _clip((A, A, 10, F32), (A, A, 10, F32)))
    _refused(ARG, lambda: _clip((A, B, 10, F32), (B + 36, B + 400, 4, F16)))
    _refused(ARG, lambda: _clip((A, A + 4, 10, F32)))
    _refused(ARG, lambda: _clip((A, B, 10, F16), (A + 400, A + 18, 4, F32)))
    need = ctc.ctc_clip_gradients_workspace_bytes(1, _gradients((A, A, 10 ** 6, F32)))
    _refused(WORKSPACE, lambda: _clip((A, A, 10 ** 6, F32), ws_bytes=need - 1))
    _refused(WORKSPACE, lambda: _clip((A, A, 10 ** 6, F32), ws=None))
    _refused(ARG, lambda: _clip((A, A, 10 ** 6, F32), ws=P + 8))
