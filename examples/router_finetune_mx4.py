"""Fine-tunes the router of a mixture-of-experts layer over frozen 4-bit experts.

The experts' weights are held in MXFP4; the router starts out skewed, so a few
experts get most of the tokens. Each step runs the layer (gate, histogram,
dispatch positions, MXFP4 expert FFN reading the routed rows, combine), takes the
mean squared distance of its output from the original layer's plus the balance
and z losses of the router, and follows the gradient back: combine -> gate
weights, losses and gate weights -> logits, logits -> router weights and bias.

    python examples/router_finetune_mx4.py [--steps N] [--tokens T] [--balance C]
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2606_00735_amd as moe  # noqa: E402


def make_layer(H, I, E, skew, seed=0):
    """Router (fp32 master weights and bias) and MXFP4 experts."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)

    def w(rows, cols):
        m = torch.randn((E, rows, cols), generator=g, device="cuda") / cols ** 0.5
        return moe.moe_mx4_quantize(m.bfloat16())

    router = torch.randn((E, H), generator=g, device="cuda") / H ** 0.5
    bias = -skew * torch.log(torch.arange(E, device="cuda") + 1.0)
    return router, bias, (w(I, H), w(I, H), w(H, I))


def forward(x, router, bias, experts, k, bufs):
    """One pass of the layer; everything the backward pass needs."""
    T, H = x.shape
    E = router.shape[0]
    emap = np.arange(E, dtype=np.int32)
    wr = router.bfloat16()
    ids, weights, logits = moe.moe_gate_topk(x, wr, bias, k, logits=True)
    counts, offsets, hws = moe.moe_expert_histogram_scan(ids, E, emap)
    _, perm_src, dest = moe.moe_permute(x, ids, emap, hws, gather=False)
    y, bufs["ffn"] = moe.moe_grouped_swiglu_ffn_mx4(moe.moe_mx4_quantize(x), *experts, offsets, perm_src=perm_src, k=k,
                                                    experts=E, ws=bufs.get("ffn"))
    out = moe.moe_unpermute_combine(y, weights, dest, T)
    return dict(wr=wr, ids=ids, weights=weights, logits=logits, counts=counts, dest=dest, y=y, out=out)


def train(steps=60, T=1024, H=1024, I=512, E=32, k=4, skew=1.0, balance=0.05, zloss=1e-4, lr=0.02, seed=0, report=None):
    """Returns (first, last): dicts of the task loss, the balance loss and the largest
    expert's load over the mean."""
    router, bias, experts = make_layer(H, I, E, skew, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1)
    x = torch.randn((T, H), generator=g, device="cuda").bfloat16()
    bufs, log = {}, []
    target = forward(x, router, bias, experts, k, bufs)["out"].float()
    scale = float(target.square().mean())
    dloss = torch.tensor([balance, zloss], device="cuda")
    m = [torch.zeros_like(router), torch.zeros_like(bias)]  # Adam's moments
    v = [torch.zeros_like(router), torch.zeros_like(bias)]
    for step in range(steps + 1):
        f = forward(x, router, bias, experts, k, bufs)
        losses, counts, live, bufs["loss"] = moe.moe_balance_loss(f["logits"], f["ids"], ws=bufs.get("loss"))
        diff = f["out"].float() - target
        log.append(dict(step=step, task=float(diff.square().mean()) / scale, balance=float(losses[0]),
                        load=float(counts.max()) * E / (T * k)))
        if report and (step % 10 == 0 or step == steps):
            report(log[-1])
        if step == steps:
            break
        dout = (2.0 / (scale * diff.numel()) * diff).bfloat16()
        dweights, _ = moe.moe_combine_backward(dout, f["y"], f["weights"], f["dest"], need_dy=False)
        dlogits = moe.moe_gate_backward(f["logits"], f["ids"], counts, live, dloss, weights=f["weights"], dweights=dweights)
        _, dw, dbias, bufs["grad"] = moe.moe_router_grad(dlogits, x, f["wr"], ws=bufs.get("grad"), need_dx=False)
        for p, d, a, b in zip((router, bias), (dw, dbias), m, v):
            a.mul_(0.9).add_(d, alpha=0.1)
            b.mul_(0.99).addcmul_(d, d, value=0.01)
            c1, c2 = 1 - 0.9 ** (step + 1), 1 - 0.99 ** (step + 1)
            p.add_(-lr * (a / c1) / ((b / c2).sqrt() + 1e-10))
    return log[0], log[-1]


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--tokens", type=int, default=1024)
    p.add_argument("--balance", type=float, default=0.05)
    a = p.parse_args(argv)
    print("step  task loss  balance loss  largest load / mean")
    train(steps=a.steps, T=a.tokens, balance=a.balance,
          report=lambda r: print(f"{r['step']:4d}  {r['task']:9.4f}  {r['balance']:12.4f}  {r['load']:19.2f}"))


if __name__ == "__main__":
    main()
