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


@pytest.mark.parametrize("t", [60, 500])
def test_over_inputs_in_a_graph(ops, t):
    """Captured with the copy that restores the keys, replayed with eager work
    between, on a stream of its own."""
    c = Case("f16", 2, t, t, 4, 2, 64, causal=True)
    o, lse = ops.attention(c.q, c.k, c.v, **c.kw)
    want = ops.attention_backward(c.do, c.q, c.k, c.v, o, lse, **c.kw)
    k, v, dq = c.k.clone(), c.v.clone(), torch.empty_like(c.q)

    def once():
        k.copy_(c.k)
        v.copy_(c.v)
        ops.attention_backward(c.do, c.q, k, v, o, lse, out=(dq, k, v), **c.kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    for _ in range(4):
        for x in (dq, k, v):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((dq, k, v), want):
            assert torch.equal(a, b)
        ops.attention_backward(c.do, c.q, c.k, c.v, o, lse, **c.kw)
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_broadcast_inputs(ops, dtype):
    """One query for all sequences, keys and values of one sequence for all, a
    value for all tokens: strides of zero, whose span is a part's."""
    c = Case(dtype, 3, 5, 300, 4, 2, 64)
    q, k = c.q[:1].expand(c.q.shape), c.k[:1].expand(c.k.shape)
    v = c.v[:, :1].expand(c.v.shape)
    for a in ((q, c.k, c.v), (c.q, k, c.v), (c.q, k, v), (q, k, v)):
        plain = [x.contiguous() for x in a]
        o, lse = ops.attention(*a)
        want = ops.attention(*plain)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
        for x, y in zip(ops.attention_backward(c.do, *a, o, lse),
                        ops.attention_backward(c.do, *plain, o, lse)):
            assert torch.equal(x, y)


def test_two_streams_at_once(ops):
    """Calls that need workspaces, under way together."""
    cases = [Case("f16", 1, 200, 7000, 2, 1, 64, seed=3 + i) for i in range(2)]
    want = []
    for c in cases:
        o, lse = ops.attention(c.q, c.k, c.v)
        want.append((o, lse) + ops.attention_backward(c.do, c.q, c.k, c.v, o, lse))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = [[] for _ in cases]
    for _ in range(10):
        for i, c in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                o, lse = ops.attention(c.q, c.k, c.v)
                got[i].append((o, lse) + ops.attention_backward(c.do, c.q, c.k, c.v, o, lse))
    torch.cuda.synchronize()
    for i, w in enumerate(want):
        for g in got[i]:
            for a, b in zip(g, w):
                assert torch.equal(a, b)
