"""Refusals of the operators' C entry points: everything is checked before
anything is enqueued, so no GPU is needed."""

import pytest

ctc = pytest.importorskip("paper_2609_16742_amd.ctc")

P = 1 << 20                      # an address that no refused call reads
F32, F16, BF16, E4M3, E5M2 = (ctc.CTC_F32, ctc.CTC_F16, ctc.CTC_BF16,
                              ctc.CTC_E4M3, ctc.CTC_E5M2)
ARG, UNSUPPORTED, WORKSPACE = (ctc.CTC_ERR_ARG, ctc.CTC_ERR_UNSUPPORTED,
                               ctc.CTC_ERR_WORKSPACE)


def _call(f, defaults, status, **change):
    args = dict(defaults)
    assert set(change) <= set(args)
    args.update(change)
    with pytest.raises(ctc.CtcError) as e:
        f(*args.values())
    assert e.value.status == status, (change, str(e.value))


NORM = dict(dtype=F16, n=2, hw=1 << 20, c=64, groups=8, carry=0, x=P, gamma=P,
            beta=P, residual=None, eps=1e-5, act=0, y=P, mean=P, rstd=P,
            ws=P, ws_bytes=1 << 30, stream=None)
NORM_BACK = dict(dtype=F16, n=2, hw=1 << 20, c=64, groups=8, carry=0, dy=P, x=P,
                 mean=P, rstd=P, gamma=P, beta=P, residual=None, act=0, dx=P,
                 dr=None, dgamma=P, dbeta=P, ws=P, ws_bytes=1 << 30,
                 stream=None)
QUANT = dict(dtype=F16, rows=100, cols=200, x=P, ldx=200, qtype=E4M3,
             block_rows=1, transpose=0, q=P, ldq=208, scales=P, lds=100,
             stream=None)
MATMUL = dict(at=E4M3, bt=E4M3, yt=F16, m=100, n=200, k=300, a=P, lda=304,
              sa=P, ldsa=100, ab=1, b=P, ldb=304, sb=P, ldsb=2, bb=128,
              bias=None, act=0, y=P, ldy=200, ws=P, ws_bytes=1 << 30,
              stream=None)
SCORES = dict(dtype=F16, rows=4, vocab=100000, logits=P, ld=100000, targets=P,
              top_k=5, lse=P, logprob=P, entropy=P, rank=P, ids=P, tops=P,
              ws=P, ws_bytes=1 << 30, stream=None)
SCORES_BACK = dict(dtype=F16, rows=4, vocab=1000, logits=P, ld=1000,
                   targets=P, lse=P, entropy=P, g_lse=P, g_logprob=P,
                   g_entropy=P, dlogits=P + 64, ldd=1000, stream=None)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(dtype=E4M3)), (ARG, dict(dtype=9)), (ARG, dict(n=-1)),
    (ARG, dict(hw=0)), (ARG, dict(c=0)), (ARG, dict(groups=0)),
    (ARG, dict(groups=7)), (ARG, dict(act=3)), (ARG, dict(eps=-1.0)),
    (ARG, dict(eps=float("nan"))), (ARG, dict(x=None)), (ARG, dict(y=None)),
    (ARG, dict(mean=None)), (UNSUPPORTED, dict(hw=1 << 40)),
    (UNSUPPORTED, dict(n=1 << 30)), (WORKSPACE, dict(ws=None)),
    (WORKSPACE, dict(ws_bytes=8)), (ARG, dict(ws=P + 4))], ids=str)
def test_group_norm_refusals(status, change):
    _call(ctc.ctc_group_norm_forward, NORM, status, **change)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(dtype=E5M2)), (ARG, dict(groups=5)), (ARG, dict(dy=None)),
    (ARG, dict(x=None)), (ARG, dict(rstd=None)), (ARG, dict(act=-1)),
    (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws_bytes=8))], ids=str)
def test_group_norm_backward_refusals(status, change):
    _call(ctc.ctc_group_norm_backward, NORM_BACK, status, **change)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(dtype=E4M3)), (ARG, dict(qtype=F16)), (ARG, dict(rows=-1)),
    (ARG, dict(ldx=199)), (ARG, dict(block_rows=2)), (ARG, dict(x=None)),
    (ARG, dict(q=None)), (ARG, dict(scales=None)), (ARG, dict(ldq=200)),
    (ARG, dict(ldq=192)), (ARG, dict(q=P + 8)), (ARG, dict(lds=99)),
    (ARG, dict(transpose=1, ldq=96)), (ARG, dict(transpose=1, lds=199)),
    (UNSUPPORTED, dict(rows=1 << 40, lds=1 << 40))], ids=str)
def test_quantize_refusals(status, change):
    _call(ctc.ctc_fp8_quantize, QUANT, status, **change)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(at=F16)), (ARG, dict(bt=F32)), (ARG, dict(yt=E4M3)),
    (ARG, dict(m=-1)), (ARG, dict(k=-1)), (ARG, dict(ab=3)),
    (ARG, dict(bb=0)), (ARG, dict(act=7)), (ARG, dict(ldy=199)),
    (ARG, dict(a=None)), (ARG, dict(b=None)), (ARG, dict(sa=None)),
    (ARG, dict(y=None)), (ARG, dict(a=P + 8)), (ARG, dict(lda=300)),
    (ARG, dict(ldb=296)), (ARG, dict(ldsa=99)), (ARG, dict(ldsb=1)),
    (UNSUPPORTED, dict(lda=1 << 23)), (UNSUPPORTED, dict(m=1 << 40, ldsa=1 << 40))],
    ids=str)
def test_matmul_refusals(status, change):
    _call(ctc.ctc_fp8_matmul, MATMUL, status, **change)


def test_matmul_needs_the_workspace_it_names():
    need = ctc.ctc_fp8_matmul_workspace_bytes(F16, 4, 64, 25088, 128)
    assert need > 0
    base = dict(MATMUL, m=4, n=64, k=25088, lda=25088, ldb=25088)
    _call(ctc.ctc_fp8_matmul, base, WORKSPACE, ws=None)
    _call(ctc.ctc_fp8_matmul, base, WORKSPACE, ws_bytes=need - 1)
    _call(ctc.ctc_fp8_matmul, base, ARG, ws=P + 8)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(dtype=E4M3)), (ARG, dict(rows=-1)), (ARG, dict(vocab=0)),
    (ARG, dict(ld=99999)), (ARG, dict(top_k=-1)), (ARG, dict(top_k=33)),
    (ARG, dict(logits=None)), (ARG, dict(targets=None)),
    (ARG, dict(ids=None)), (ARG, dict(tops=None)),
    (UNSUPPORTED, dict(rows=1 << 40)), (WORKSPACE, dict(ws=None)),
    (WORKSPACE, dict(ws_bytes=8)), (ARG, dict(ws=P + 8))], ids=str)
def test_token_scores_refusals(status, change):
    _call(ctc.ctc_token_scores_forward, SCORES, status, **change)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(dtype=E5M2)), (ARG, dict(ldd=999)), (ARG, dict(logits=None)),
    (ARG, dict(lse=None)), (ARG, dict(dlogits=None)),
    (ARG, dict(targets=None)), (ARG, dict(entropy=None)),
    (ARG, dict(dlogits=P, ldd=1001))], ids=str)
def test_token_scores_backward_refusals(status, change):
    _call(ctc.ctc_token_scores_backward, SCORES_BACK, status, **change)


def test_empty_calls_do_nothing():
    ctc.ctc_group_norm_forward(*dict(NORM, n=0, x=None, y=None, ws=None,
                                     ws_bytes=0).values())
    ctc.ctc_fp8_quantize(*dict(QUANT, rows=0, x=None, q=None,
                               scales=None).values())
    ctc.ctc_fp8_matmul(*dict(MATMUL, m=0, a=None, y=None, sa=None, ws=None,
                             ws_bytes=0).values())
    ctc.ctc_token_scores_forward(*dict(SCORES, rows=0, logits=None, ws=None,
                                       ws_bytes=0).values())
    ctc.ctc_token_scores_backward(*dict(SCORES_BACK, rows=0, logits=None,
                                        dlogits=None).values())


def test_the_networks_refuse_the_operators_types():
    d = ctc.layer_desc(16, 16, 3, 3, 1, 1, 1, 0, ctc.CTC_ROLE_NONE)
    for dt in (BF16, E4M3, E5M2):
        with pytest.raises(ctc.CtcError) as e:
            ctc.ctc_conv2d_workspace_bytes(d, dt, 1, 8, 8)
        assert e.value.status == ARG


def test_group_norm_takes_many_images():
    """n * c below 2^32 (and no less) is taken, whatever the map's size."""
    for n, hw, c in [(4093, 1, 512), (4094, 1, 16), (10000, 4, 64), (1 << 20, 1, 2048),
                     ((1 << 31) - 1, 1, 2), (1 << 24, 1 << 20, 255), (5, 1 << 31, 24)]:
        for backward in (0, 1):
            for dtype in (F32, F16, BF16):
                ctc.ctc_group_norm_workspace_bytes(dtype, n, hw, c, 1, backward)
    for n, c in [(1 << 16, 1 << 16), (1 << 30, 4)]:
        for f, base in ((ctc.ctc_group_norm_forward, NORM),
                        (ctc.ctc_group_norm_backward, NORM_BACK)):
            _call(f, base, UNSUPPORTED, n=n, c=c, groups=4)


def test_the_limits_that_the_header_names():
    """Sizes at the limit are taken, one more is refused."""
    mm = ctc.ctc_fp8_matmul_workspace_bytes
    sc = ctc.ctc_token_scores_workspace_bytes
    for f, at, past in [
            (mm, (F16, 2 ** 21, 4091, 128, 128), (F16, 2 ** 21, 4092, 128, 128)),
            (mm, (F16, 1, 2 ** 23 - 2, 128, 128), (F16, 1, 2 ** 23 - 1, 128, 128)),
            (mm, (F16, 2 ** 30, 1, 128, 128), (F16, 2 ** 30 + 1, 1, 128, 128)),
            (sc, (2 ** 22 - 1, 4096, 0), (2 ** 22, 4096, 0)),
            (sc, (1, 2 ** 30, 1), (1, 2 ** 30 + 1, 1))]:
        f(*at)
        with pytest.raises(ctc.CtcError) as e:
            f(*past)
        assert e.value.status == UNSUPPORTED, past
    base = dict(QUANT, rows=16 * (2 ** 22 - 1), cols=128, ldx=128, ldq=128, lds=2 ** 30)
    # (2^22 rows / 16 by 2: past it; one row less gets to the NULL matrix)
    _call(ctc.ctc_fp8_quantize, base, UNSUPPORTED)
    _call(ctc.ctc_fp8_quantize, base, ARG, rows=16 * (2 ** 22 - 1) - 1, q=None)
