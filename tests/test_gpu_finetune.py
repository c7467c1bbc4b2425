"""The head trained on a protected network's features: its gradients against
64-bit autograd of the formulas, and a run on a network's own features."""

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def finetune():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import finetune
    return finetune


def _reference(head, x, targets, out):
    """Gradients in 64 bits at the logits of `out` (the 8-bit products moved
    them, and the softmax's gradient with them), with the magnitudes of the
    terms of both products of the linear layer."""
    x = x.double()
    n, c = x.shape[0], x.shape[-1]
    per = c // head.groups
    v = x.flatten(1, -2).view(n, -1, head.groups, per)
    use = torch.ones((head.groups, per), dtype=torch.float64, device=x.device)
    use[-1, -1] = 0
    count = use.sum(1) * v.shape[1]
    mean = (v * use).sum((1, 3)) / count
    d = v - mean[:, None, :, None]
    var = (d * d * use).sum((1, 3)) / count
    xhat = (d / torch.sqrt(var + 1e-5)[:, None, :, None]).view(n, -1, c)
    z = xhat * head.gamma.double() + head.beta.double()
    pooled = z.clamp(min=0).mean(1)[:, :-1]
    logits = out[:, :-1].double()
    dl = torch.softmax(logits, 1)
    dl[torch.arange(n, device=x.device), targets.long()] -= 1
    w = head.weight.double()
    dz = torch.zeros_like(z)
    dz[..., :-1] = (z[..., :-1] > 0) * (dl @ w)[:, None]
    size = torch.zeros_like(z)
    size[..., :-1] = (z[..., :-1] > 0) * (dl.abs() @ w.abs())[:, None]
    return {"gamma": ((dz * xhat).sum((0, 1)), (size * xhat.abs()).sum((0, 1))),
            "beta": (dz.sum((0, 1)), size.sum((0, 1))),
            "weight": (dl.t() @ pooled, dl.abs().t() @ pooled),
            "bias": (dl.sum(0), dl.abs().sum(0)),
            "logits": (pooled @ w.t(), pooled @ w.t().abs())}


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_head_gradients(finetune, dtype):
    """A value in 8 bits is off by 2^-4 (e4m3) or 2^-3 (e5m2) of itself, or,
    where it is small against its block's largest, by 2^-10 or 2^-17 of the
    format's scale: of the block's largest that is less than 2^-17.  A product
    of two is off by the sum of both and their product."""
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    n, c, classes = 9, 48, 21
    x = torch.randn((n, 5, 4, c), device="cuda", generator=g).to(dtype)
    x[..., -1] = x[..., -1].abs() * 40
    targets = torch.randint(0, classes, (n,), device="cuda", generator=g,
                            dtype=torch.int32)
    head = finetune.Head(c, classes, groups=8)
    head.gamma.add_(0.2 * torch.randn(c, device="cuda", generator=g))
    head.beta.add_(0.2 * torch.randn(c, device="cuda", generator=g))
    head.bias.add_(0.1 * torch.randn(classes, device="cuda", generator=g))
    out, saved = head.forward(x)
    logprob, dgamma, dbeta, dw, db = head.gradients(out, targets, saved)
    want = _reference(head, x, targets, out)
    e4, e5 = 2.0 ** -4, 2.0 ** -3
    both, same = e4 + e5 + e4 * e5, 2 * e4 + e4 * e4
    # (a map of 16 bits: 2^-11 of the gradient, and of the pooled values)
    rest = 2.0 ** -9
    got = {"gamma": (dgamma, both), "beta": (dbeta, both), "weight": (dw, both),
           "bias": (db, 0.0), "logits": (out[:, :-1] - head.bias, same)}
    for k, (v, e) in got.items():
        w, size = want[k]
        off = (v.double() - w).abs()
        assert bool((off <= (e + rest) * size + 2.0 ** -12 * size.max()).all()), k
    lp = torch.log_softmax(out[:, :-1].double(), 1).gather(
        1, targets.long()[:, None])[:, 0]
    assert float((logprob.double() - lp).abs().max()) <= 2.0 ** -20 * float(
        1 + lp.abs().max())
    # the checksum passes: its mean over the pixels closes the row
    s = x[..., -1].double().mean((1, 2))
    assert float((out[:, -1].double() - s).abs().max()) <= 2.0 ** -20 * float(s.max())
    assert float(dgamma[-1]) == 0 and float(dbeta[-1]) == 0


@pytest.mark.parametrize("workload,c", [("resnet20_f32_b128", 64),
                                        ("resnet18_f16_b64", 512)])
def test_features_are_the_last_map(finetune, workload, c):
    """Its mean over the pixels is what the network's own pool computes."""
    from paper_2609_16742_amd import CtcNet
    from workloads import config, gen
    w = config(workload)
    net = CtcNet(w.layers, w.in_shape, w.classes, w.dtype, gen.make_params(w),
                 max_batch=4)
    x = torch.from_numpy(gen.make_inputs(w, 4)).cuda()
    f = finetune.features(net, x)
    assert f.shape[0] == 4 and f.shape[-1] == c
    gap = next(i for i, l in enumerate(w.layers) if l["op"] == "gap")
    pooled = net.tensor(gap + 1, 4).flatten(1)[:, :c].double()
    want = f.double().flatten(1, 2).mean(1)
    u = 2.0 ** -10 if w.dtype == "f16" else 2.0 ** -18
    assert bool(((pooled - want).abs() <= u * want.abs().max()).all())


def test_training_on_a_protected_network(finetune):
    r = finetune.run("resnet20_f32_b128", classes=10, steps=60, lr=0.5)
    # log 10 at the start, up to the first weights' noise
    assert abs(r["loss_first"] - np.log(10)) < 1.5
    assert r["loss_last"] < r["loss_first"]
    assert r["flagged"] <= 2             # alpha = 0.01 of 128
