"""Reading a protected network's features leaves the network as it was."""

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("workload", ["resnet20_f32_b128", "resnet18_f16_b64",
                                      "mobilenetv2_f16_b128"])
@pytest.mark.parametrize("kinds", [None, 0, 12])
def test_features_keep_the_networks_fusions(workload, kinds):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import CtcNet, ctc, finetune
    from workloads import config, gen
    w = config(workload)
    net = CtcNet(w.layers, w.in_shape, w.classes, w.dtype, gen.make_params(w), max_batch=8)
    if kinds is not None:
        net.set_fusion(kinds)

    def kernels():
        return [ctc.ctc_net_op_kernel(net.h, i, 8) for i in range(len(w.layers))]
    x = torch.from_numpy(gen.make_inputs(w, 8)).cuda()
    before, out = kernels(), net.forward(x)
    f = finetune.features(net, x)
    assert bool(torch.isfinite(f.float()).all())
    assert kernels() == before
    assert torch.equal(net.forward(x), out)


def test_head_trains_like_its_64_bit_form():
    """40 steps of gradient descent against the same steps in 64 bits with
    autograd's gradients.  A product's operands are off by 2^-4 and 2^-3 of
    themselves at most, so a step's gradient by less than a fifth of what it
    is a sum of; a wrong scale or a missing part is more than that."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import finetune, ops
    n, c, classes, groups, lr = 96, 64, 10, 8, 0.5
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    x = torch.randn((n, 5, 5, c), device="cuda", generator=g) + torch.randn(
        (n, 1, 1, c), device="cuda", generator=g)
    x[..., -1] = 20 * x[..., -1].abs()
    t = torch.randint(0, classes, (n,), device="cuda", generator=g, dtype=torch.int32)
    head = finetune.Head(c, classes, groups=groups)
    p = [v.double().requires_grad_() for v in (head.gamma, head.beta, head.weight, head.bias)]
    per = c // groups
    v = x.double().view(n, -1, groups, per)
    use = torch.ones((groups, per), dtype=torch.float64, device="cuda")
    use[-1, -1] = 0
    count = use.sum(1) * v.shape[1]
    mean = ((v * use).sum((1, 3)) / count)[:, None, :, None]
    var = ((v - mean).square() * use).sum((1, 3)) / count
    xhat = ((v - mean) / torch.sqrt(var + 1e-5)[:, None, :, None]).view(n, -1, c)

    def loss():
        z = (xhat * p[0] + p[1]).clamp(min=0).mean(1)[:, :-1]
        logits = z @ p[2].t() + p[3]
        return torch.nn.functional.cross_entropy(logits, t.long()), logits
    first = [float(loss()[0].detach()), float(head.step(x, t, lr))]
    for i in range(40):
        for q, d in zip(p, torch.autograd.grad(loss()[0], p)):
            q.data.sub_(d, alpha=lr)
        if i:                                    # (one is done)
            head.step(x, t, lr)
    want, logits = loss()
    s = ops.token_scores(head.forward(x)[0][:, :-1], t)
    fall = [first[0] - float(want.detach()), first[1] + float(s.logprob.mean())]
    assert abs(first[1] - first[0]) <= 0.02 * first[0], first
    assert fall[0] > 0.3 and abs(fall[1] - fall[0]) <= 0.2 * fall[0], fall
    right = [int((logits.argmax(1) == t).sum()), int((s.rank == 0).sum())]
    assert right[0] >= n // 2 and abs(right[1] - right[0]) <= n // 10, right
    for q, own in zip(p, (head.gamma, head.beta, head.weight, head.bias)):
        start = torch.ones_like(q) if q is p[0] else torch.zeros_like(q)
        if q is p[2]:
            start = finetune.Head(c, classes, groups=groups).weight.double()
        moved = (q - start).detach()
        assert float((own.double() - start - moved).norm()) <= 0.2 * float(moved.norm())


@pytest.mark.parametrize("dims", [(), (1,), (6,), (2, 3)])
def test_head_takes_maps_of_any_dimensions(dims):
    """[n, c] rows of features among them: the same numbers as [n, 1, .., c]."""
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_16742_amd import finetune
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = torch.randn((5,) + dims + (32,), device="cuda", generator=g)
    t = torch.arange(5, device="cuda", dtype=torch.int32)
    whole = x.view(5, 1, -1, 32)
    heads = [finetune.Head(32, 7, groups=4) for _ in range(2)]
    loss = [h.step(v, t, 0.5) for h, v in zip(heads, (x, whole))]
    assert torch.equal(*loss)
    for name in ("gamma", "beta", "weight", "bias"):
        assert torch.equal(getattr(heads[0], name), getattr(heads[1], name)), name
    assert torch.equal(heads[0].answers(x).top_ids, heads[1].answers(whole).top_ids)
