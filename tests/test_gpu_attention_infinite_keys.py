"""Infinite keys among causal queries.

A key whose score is -infinity has a probability of zero: it is a key that is
far from a query, but for its product with ds = 0 in dq, 0 times infinity, a NaN
in the column where it is infinite.  So results are the bits of those with a key
that is merely far (its probability underflows to zero), and that column shows a
NaN for the queries that see it.  A score of +infinity makes the query's results
NaN."""

import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_attention import DT, Case  # noqa: E402

INF = math.inf


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import ops
    return ops


# queries and keys that one workgroup takes, several tiles, few queries over
# ranges of many keys
SHAPES = [(50, 50, 64), (64, 64, 128), (30, 40, 32), (200, 200, 64), (200, 200, 128),
          (333, 400, 96), (70, 4000, 64), (70, 4000, 128)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_infinite_key(ops, shape, sign, dtype):
    tq, tk, d = shape
    far = {"f16": 60000.0, "bf16": 1e30}[dtype]
    e = 5
    # (heads 0 and 1 share key head 0)
    c = Case(dtype, 2, tq, tk, 4, 2, d, causal=True)
    shift = tk - tq
    for j in (shift, shift + 1, shift + tq // 2, tk - 2, tk - 1, tk // 3):
        after = slice(max(0, j - shift), tq)
        before = slice(0, max(0, j - shift))

        def run(value, second):
            q, k = c.q.clone(), c.k.clone()
            q[0, :, 0, e], q[0, :, 1, e] = sign, sign * second
            k[0, j, 0, e] = value
            o, lse = ops.attention(q, k, c.v, causal=True)
            g = ops.attention_backward(c.do, q, k, c.v, o, lse, causal=True)
            return dict(zip(("o", "lse", "dq", "dk", "dv"), (o, lse.transpose(1, 2)) + g))
        # the query that sees this key alone has a softmax of nothing
        alone = [j - shift] if j == 0 else []
        want, got = run(-sign * far, 1), run(-sign * INF, 1)
        rows = [i for i in range(tq) if i not in alone]
        for n in ("o", "lse"):
            assert torch.equal(got[n][:, rows], want[n][:, rows]), n
        keep = [i for i in range(d) if i != e]
        assert torch.equal(got["dq"][:, rows][..., keep], want["dq"][:, rows][..., keep])
        assert torch.equal(got["dq"][1], want["dq"][1])
        assert torch.equal(got["dq"][0, :, 2:], want["dq"][0, :, 2:])
        assert torch.equal(got["dq"][0, before], want["dq"][0, before])
        assert bool(torch.isnan(got["dq"][0, after, :2, e]).all())
        # one head with +infinity
        got = run(-sign * INF, -1)
        for n in ("o", "lse", "dq"):
            a, b = got[n][0], want[n][0]
            assert torch.equal(a[before, 0], b[before, 0]), n
            assert bool(torch.isnan(a[after, 1]).all()), n
            assert bool(torch.isfinite(a[before, 1].float()).all()) or n == "lse", n
        assert torch.equal(got["dq"][0, rows, 0][:, keep], want["dq"][0, rows, 0][:, keep])


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients_of_an_infinite_key(ops, shape, causal, dtype):
    """Those of the key itself: no query has a part in it, nor has a row of a
    tile behind the last query."""
    tq, tk, d = shape
    e, j = 5, tk - tq + 3
    c = Case(dtype, 2, tq, tk, 4, 2, d, causal=causal, q_lengths=[tq, tq - 2],
             k_lengths=[tk, tk - 2])
    q, k = c.q.clone(), c.k.clone()
    q[..., :2, e] = 1

    def run(value):
        k[:, j, 0, e] = value
        o, lse = ops.attention(q, k, c.v, **c.kw)
        return (o, lse) + ops.attention_backward(c.do, q, k, c.v, o, lse, **c.kw)
    want = run({"f16": -60000.0, "bf16": -1e30}[dtype])
    got = run(-INF)
    for i in (0, 1, 3, 4):
        assert torch.equal(got[i], want[i]), i
    assert not got[3][:, j, 0].any() and not got[4][:, j, 0].any()
    keep = [i for i in range(d) if i != e]
    assert torch.equal(got[2][..., keep], want[2][..., keep])
