"""Attention whose results are written over its inputs, where that is allowed:
the bits of results of their own."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import DT, Case  # noqa: E402


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import ops
    return ops


# a workgroup's keys and rows, many of both, ranges of keys, ranges of rows,
# both, heads that share keys; every width of kernel
SHAPES = [(3, 50, 60, 4, 2, 64), (1, 64, 64, 2, 2, 128), (2, 500, 700, 4, 4, 64),
          (1, 900, 1100, 6, 2, 128), (1, 70, 9000, 2, 1, 96), (1, 3000, 60, 4, 1, 32),
          (1, 600, 600, 1, 1, 80)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_over_inputs(ops, shape, causal, dtype):
    c = Case(dtype, *shape, causal=causal)
    o, lse = ops.attention(c.q, c.k, c.v, **c.kw)
    q = c.q.clone()
    o2, lse2 = ops.attention(q, c.k, c.v, out=(q, torch.empty_like(lse)), **c.kw)
    assert torch.equal(o2, o) and torch.equal(lse2, lse) and o2.data_ptr() == q.data_ptr()

    def backward(k, v, over):
        k, v = (k.clone(), v.clone()) if v is not k else (k.clone(),) * 2
        t = {"q": torch.empty_like(c.q), "k": k, "v": v, "x": torch.empty_like(k),
             "y": torch.empty_like(v)}
        return ops.attention_backward(c.do, c.q, k, v, o, lse,
                                      out=tuple(t[n] for n in "q" + over), **c.kw)
    want = backward(c.k, c.v, "xy")
    for over in ("ky", "xv", "kv", "vk", "vy", "xk"):
        for a, b in zip(backward(c.k, c.v, over), want):
            assert torch.equal(a, b), over
    # values that are the keys
    o, lse = ops.attention(c.q, c.k, c.k, **c.kw)
    want = backward(c.k, c.k, "xy")
    for over in ("ky", "xk"):
        for a, b in zip(backward(c.k, c.k, over), want):
            assert torch.equal(a, b), over


def test_refusals(ops):
    from paper_2609_16742_amd import ctc
    x = torch.zeros((1, 8, 12, 64), device="cuda", dtype=DT["f16"])
    q, k, v = x[:, :, :4], x[:, :, 4:8], x[:, :, 8:]
    o, lse = ops.attention(q, k, v)
    dq, dk, dv = (torch.empty_like(t) for t in (q, k, v))
    for out in ((q, dk, dv), (k, dk, dv), (o, dk, dv), (dq, q, dv), (dq, dk, dk), (dq, dv, dv),
                (dq, x[:, :, 3:7], dv), (dq, dk, x[:, :, 5:9])):
        with pytest.raises(ctc.CtcError):
            ops.attention_backward(o, q, k, v, o, lse, out=out)
    for out in ((k, lse), (v, lse), (x[:, :, 1:5], lse)):
        with pytest.raises(ctc.CtcError):
            ops.attention(q, k, v, out=out)
    assert not x.any()
