"""Trains a new classifier on the features of a protected network.

A protected network (:class:`CtcNet`) runs as deployed; its last feature map
[n, h, w, c], whose last channel is the carry-through checksum, goes into a
small head:

    group norm and ReLU (the checksum passes) -> mean over the pixels
    -> 8-bit product with the head's filters -> scores of the right classes

Rows of the head's output end with the pooled checksum, like those of a
protected classifier, so :func:`ctc.ctc_verify` checks them.  The backward
pass takes the same operators the other way: gradient of the scores, both
8-bit products of the linear layer, gradient of the group norm.

    python -m paper_2609_16742_amd.finetune --workload resnet18_f16_b64
"""

from __future__ import annotations

import argparse
import json
import sys
import time

import torch

from . import ctc, ops
from .runtime import CtcNet


class Head:
    """Group norm, ReLU, mean over the pixels and a linear layer of
    ``classes`` outputs on maps of ``channels`` channels, the last of them
    the checksum.  Parameters are fp32; the products run in 8 bits."""

    def __init__(self, channels, classes, groups=32, seed=0, device="cuda"):
        if channels < 2 or channels % groups:
            raise ValueError("groups do not divide the channels")
        self.groups, self.classes = groups, classes
        g = torch.Generator().manual_seed(seed)
        self.gamma = torch.ones(channels, device=device)
        self.beta = torch.zeros(channels, device=device)
        self.weight = (torch.randn((classes, channels - 1), generator=g)
                       / (channels - 1) ** 0.5).to(device)
        self.bias = torch.zeros(classes, device=device)

    def forward(self, x):
        """([n, classes + 1] fp32 logits and pooled checksum, what
        :meth:`gradients` needs of the pass) for a map x [n, ..., c]."""
        y, mean, rstd = ops.group_norm(x, self.groups, self.gamma, self.beta,
                                       act="relu", carry=True)
        pooled = y.view(y.shape[0], -1, y.shape[-1]).mean(
            1, dtype=torch.float32)
        out = torch.empty((x.shape[0], self.classes + 1), device=x.device)
        out[:, -1] = pooled[:, -1]
        pooled = pooled[:, :-1]          # rows keep their stride
        qa, sa = ops.fp8_quantize(pooled)
        qw, sw = ops.fp8_quantize(self.weight, block_rows=128)
        ops.fp8_matmul(qa, sa, qw, sw, self.bias, out=out[:, :-1])
        return out, (x, mean, rstd, pooled)

    def gradients(self, out, targets, saved):
        """(log probabilities [n], gradients of minus their sum with respect
        to gamma, beta, weight and bias; gamma's and beta's times the
        pixels)."""
        x, mean, rstd, pooled = saved
        logits = out[:, :-1]
        s = ops.token_scores(logits, targets)
        minus = torch.full_like(s.lse, -1.0)
        d = ops.token_scores_backward(logits, targets, s.lse, g_logprob=minus)
        # weight: d^T pooled; pooled: d weight
        qd, sd = ops.fp8_quantize(d, "e5m2", transpose=True)
        qp, sp = ops.fp8_quantize(pooled, transpose=True)
        dw = ops.fp8_matmul(qd, sd, qp, sp, dtype=torch.float32)
        qd, sd = ops.fp8_quantize(d, "e5m2")
        qw, sw = ops.fp8_quantize(self.weight, block_rows=128, transpose=True)
        dp = ops.fp8_matmul(qd, sd, qw, sw, dtype=torch.float32)
        # every pixel gets dp (over the pixels: left to the caller, so that
        # 16-bit gradients do not vanish); the checksum gets none
        dy = torch.zeros_like(x)
        dy[..., :-1] = dp.view((dp.shape[0],) + (1,) * (x.dim() - 2) + (-1,))
        _, _, dgamma, dbeta = ops.group_norm_backward(
            dy, x, mean, rstd, self.groups, self.gamma, self.beta, act="relu",
            carry=True, out=(None, None, torch.empty_like(self.gamma),
                             torch.empty_like(self.beta)))
        return s.logprob, dgamma, dbeta, dw, d.sum(0)

    def step(self, x, targets, lr):
        """One step of gradient descent on the mean of -log p(target);
        returns that mean (a tensor; nothing waits)."""
        out, saved = self.forward(x)
        logprob, dgamma, dbeta, dw, db = self.gradients(out, targets, saved)
        n, pixels = x.shape[0], x[0, ..., 0].numel()
        self.gamma.sub_(dgamma, alpha=lr / (n * pixels))
        self.beta.sub_(dbeta, alpha=lr / (n * pixels))
        self.weight.sub_(dw, alpha=lr / n)
        self.bias.sub_(db, alpha=lr / n)
        return -logprob.mean()

    def answers(self, x, k=5):
        """TokenScores of the ``k`` best classes of every row."""
        return ops.token_scores(self.forward(x)[0][:, :-1], None,
                                min(k, self.classes))


def features(net, x):
    """The protected network's last feature map [n, h, w, c] for images x
    (what its global pool or its first FC layer reads); valid until the
    network's next pass.  This pass fuses no residual blocks; the kinds of
    :meth:`CtcNet.set_fusion` stay in effect for others."""
    if net.mode != 1:
        raise ValueError("a network protected in replace mode is needed")
    # (a block fused with the classifier would not store the map)
    chosen = net.fusion
    net.set_fusion(chosen & ~ctc.CTC_FUSE_BLOCK)
    try:
        net.forward(x)
    finally:
        net.set_fusion(chosen)
    i = next(i for i, l in enumerate(net.layers) if l["op"] in ("gap", "fc"))
    at = net.layers[i]["inp"]
    t = at
    while net.layers[t - 1]["op"] != "conv":
        t = net.layers[t - 1]["inp"]
    c = net.layers[t - 1]["c_out"]
    return net.tensor(at, x.shape[0])[..., :c].contiguous()


def run(workload, classes=100, steps=200, lr=0.5, log=None):
    """Fits a head to random classes of one batch of images; returns the loss
    before and after, how many classes are ranked first, how many rows the
    detector flags after calibration on them, and the time of a step."""
    from workloads import config, gen

    w = config(workload)
    net = CtcNet(w.layers, w.in_shape, w.classes, w.dtype, gen.make_params(w),
                 max_batch=w.batch)
    x = torch.from_numpy(gen.make_inputs(w, w.batch)).cuda()
    f = features(net, x)
    g = torch.Generator().manual_seed(1)
    targets = torch.randint(0, classes, (w.batch,), generator=g,
                            dtype=torch.int32).cuda()
    head = Head(f.shape[-1], classes, groups=8)
    first = float(head.step(f, targets, lr))
    torch.cuda.synchronize()
    t = time.perf_counter()
    for i in range(1, steps):
        loss = head.step(f, targets, lr)
        if log and i % 50 == 0:
            log("step %d: loss %.4f" % (i, float(loss)))
    torch.cuda.synchronize()
    ms = (time.perf_counter() - t) * 1e3 / max(1, steps - 1)
    out, _ = head.forward(f)
    s = ops.token_scores(out[:, :-1], targets, 1)
    S = out[:, -1].contiguous()
    ref, tau = ctc.ctc_threshold_from_samples(S.cpu().numpy(), 0.01)
    flags = torch.empty(w.batch, dtype=torch.uint8, device="cuda")
    count = torch.empty(1, dtype=torch.int32, device="cuda")
    ctc.ctc_verify(S, w.batch, 1, ref, tau, flags, count, None)
    return {"workload": workload, "classes": classes, "steps": steps,
            "loss_first": first, "loss_last": -float(s.logprob.mean()),
            "ranked_first": int((s.rank == 0).sum()), "images": w.batch,
            "flagged": int(count), "ms_per_step": ms}


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--workload", default="resnet18_f16_b64")
    ap.add_argument("--classes", type=int, default=100)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--lr", type=float, default=0.5)
    a = ap.parse_args(argv)
    if not torch.cuda.is_available():
        sys.exit("training runs on the GPU")
    print(json.dumps(run(a.workload, a.classes, a.steps, a.lr,
                         log=lambda s: print(s, flush=True))))


if __name__ == "__main__":
    main()
