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
