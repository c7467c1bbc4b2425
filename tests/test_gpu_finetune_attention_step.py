"""The attention head's step as a whole: the norm's gradients through attention,
and the step (gradients, clipping and update) in a graph."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_gpu_finetune_attention import _attend, _case, finetune  # noqa: E402,F401


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_gradients_of_the_norm(finetune, dtype):  # noqa: F811
    """dgamma and dbeta against 64-bit autograd of what is behind the norm, whose
    gradient goes through the 8-bit filters: 2^-3 and 2^-4 of the operands, the
    16-bit roundings in front of them 2^-7 and 2^-8 at most."""
    head, x, targets = _case(finetune, dtype)
    out, saved = head.forward(x)
    _, dp, _, _ = head._linear_gradients(out, targets, saved[-1])
    qkv = saved[4].double().requires_grad_()
    pooled = _attend(qkv, head.q_weight.double(), head.k_weight.double(), head, 6, 5)
    pixels = x.shape[1] * x.shape[2]
    d, = torch.autograd.grad((pooled * dp.double()).sum() * pixels, (qkv,))
    d = d.reshape(-1, qkv.shape[2] * qkv.shape[3])
    project = head.project.double()
    dy, ay = d @ project, d.abs() @ project.abs()
    mean, rstd = (t.double().view(x.shape[0], 1, head.groups, 1) for t in saved[1:3])
    c = x.shape[-1]
    xhat = ((x.double().view(x.shape[0], -1, head.groups, c // head.groups) - mean) * rstd)
    xhat = xhat.view(-1, c)[:, :-1]
    z = (saved[3].double() > 0).double()
    dgamma, dbeta = head._pixel_gradients(dp, saved)[:2]
    e = 2.0 ** -3 + 2.0 ** -4 + 2.0 ** -7 + 2.0 ** -8
    for got, part in ((dgamma, z * xhat), (dbeta, z)):
        want, size = (dy * part).sum(0), (ay * part.abs()).sum(0)
        assert bool(((got[:-1].double() - want).abs() <= e * size + 2.0 ** -10 * size.max()).all())
        # (and they are gradients, not what the bound alone would let through)
        assert float((got[:-1].double() - want).norm()) <= 0.25 * float(want.norm())


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_steps_in_a_graph(finetune, dtype):  # noqa: F811
    """Captured with its clipping and update, replayed with eager work between:
    parameters and losses of eager steps, bit for bit."""
    head, x, targets = _case(finetune, dtype)
    start = [p.clone() for p in head.parameters()]

    def reset():
        for p, v in zip(head.parameters(), start):
            p.copy_(v)
    want = []
    for i in range(5):
        loss = head.step(x, targets, 0.25, max_norm=0.5)
        want.append([loss.clone()] + [p.clone() for p in head.parameters()])
    reset()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        head.step(x, targets, 0.25, max_norm=0.5)
    torch.cuda.current_stream().wait_stream(side)
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = head.step(x, targets, 0.25, max_norm=0.5)
    for p, v in zip(head.parameters(), start):
        assert torch.equal(p, v)
    for values in want:
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip([loss] + head.parameters(), values):
            assert torch.equal(a, b)
        out, _ = head.forward(x)
        assert bool(torch.isfinite(out).all())
        torch.cuda.synchronize()
    moved = [float((a - b).abs().max()) for a, b in zip(head.parameters(), start)]
    assert min(moved) > 0
