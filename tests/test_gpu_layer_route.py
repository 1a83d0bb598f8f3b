"""GPU tests of moe_layer(route=...) as a program calls it: bf16 and fp32, sizes of the
library's workloads, the fused gather, boolean masks, a caller's buffer for the logits. Its outputs
are those of its own steps called one by one, so they are compared bit for bit; ids and weights are the oracle's on the logits that it used."""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16
ROUTE = {"score": "sigmoid", "n_group": 4, "topk_group": 2, "norm": True, "scale": 2.5}


def make(T, H, I, E, dtype, seed=3, local=None):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def n(*shape):
        return (torch.randn(shape, generator=g, device=DEV) / shape[-1] ** 0.5).to(dtype)

    local = E if local is None else local
    emap = np.full(E, -1, np.int32)
    emap[:local] = np.arange(local)
    return {"x": n(T, H) * H ** 0.5, "wr": n(E, H), "bias": torch.randn(E, generator=g, device=DEV) / 10, "emap": emap,
            "wg": n(local, I, H), "wu": n(local, I, H), "wd": n(local, H, I)}


def layer(t, k, **kw):
    return moe.moe_layer(t["x"], t["wr"], t["bias"], k, t["emap"], t["wg"], t["wu"], t["wd"], **kw)


def steps(t, k, route, fuse_gather=False):
    _, _, logits = moe.moe_gate_topk(t["x"], t["wr"], None, 1, logits=True)
    ids, w = moe.moe_route(logits, k, bias=t["bias"], **route)
    counts, offsets, ws = moe.moe_expert_histogram_scan(ids, t["wr"].shape[0], t["emap"])
    xp, src, dest = moe.moe_permute(t["x"], ids, t["emap"], ws, gather=not fuse_gather)
    if fuse_gather:
        y, _ = moe.moe_grouped_swiglu_ffn_gather(t["x"], src, k, t["wg"], t["wu"], t["wd"], offsets, experts=t["wr"].shape[0])
    else:
        y, _ = moe.moe_grouped_swiglu_ffn(xp, t["wg"], t["wu"], t["wd"], offsets)
    return {"logits": logits, "ids": ids, "weights": w, "counts": counts, "offsets": offsets, "dest": dest,
            "out": moe.moe_unpermute_combine(y, w, dest, t["x"].shape[0])}


# tokens, H, I, experts, of these on this GPU, k, type
SIZES = [(1, 2048, 768, 128, 128, 8, BF), (97, 2048, 768, 128, 128, 8, BF), (130, 7168, 2048, 256, 8, 8, BF),
         (64, 5120, 8192, 16, 2, 2, BF), (48, 128, 256, 8, 8, 2, torch.float32)]


@pytest.mark.parametrize("T,H,I,E,local,k,dtype", SIZES)
def test_layer_is_its_steps(T, H, I, E, local, k, dtype):
    print("CASE routed layer", T, H, I, E, k, dtype, flush=True)
    t = make(T, H, I, E, dtype, local=local)
    mask = torch.ones(T, dtype=torch.uint8, device=DEV)
    if T > 1:
        mask[T - 3:] = 0
    for route in (ROUTE, {"score": "softmax", "norm": False}, {**ROUTE, "mask": mask}):
        r, want = layer(t, k, route=route), steps(t, k, route)
        for n, v in want.items():
            assert torch.equal(r[n], v), n
        plain = {n: v for n, v in route.items() if n != "mask"}
        ids, w = O.route(r["logits"].cpu().numpy(), k, bias=t["bias"].double().cpu().numpy(),
                         mask=mask.cpu().numpy() if "mask" in route else None, **plain)
        assert np.array_equal(r["ids"].cpu().numpy(), ids)
        assert np.allclose(r["weights"].cpu().numpy(), w, rtol=1e-5, atol=0)
        if dtype == BF:
            fused = layer(t, k, route=route, fuse_gather=True)
            assert fused["x_perm"] is None
            # its own steps: the FFN that gathers may sum in another order than the one that does not
            for n, v in steps(t, k, route, fuse_gather=True).items():
                assert torch.equal(fused[n], v), n
        if "mask" in route and T > 1:
            assert (r["ids"][T - 3:] == -1).all() and (r["out"][T - 3:] == 0).all()


def test_boolean_masks():
    """As moe_balance_loss and moe_gate_backward take them."""
    print("CASE routed layer bool mask", flush=True)
    t = make(50, 128, 256, 16, BF)
    mask = torch.arange(50, device=DEV) % 3 != 0
    as_bytes = mask.to(torch.uint8)
    z = torch.randn((50, 16), device=DEV)
    a, b = moe.moe_route(z, 4, mask=mask), moe.moe_route(z, 4, mask=as_bytes)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and (a[0][~mask] == -1).all()
    r, s = layer(t, 4, route={**ROUTE, "mask": mask}), layer(t, 4, route={**ROUTE, "mask": as_bytes})
    assert torch.equal(r["ids"], s["ids"]) and torch.equal(r["out"], s["out"])
    with pytest.raises(ValueError):
        moe.moe_route(z, 4, mask=mask[:49])
    with pytest.raises(ValueError):
        moe.moe_route(z, 4, mask=mask.int())


@pytest.mark.parametrize("bufs", [False, True])
def test_logits_go_to_the_callers_buffer(bufs):
    """As without route: logits may be a tensor that receives them."""
    print("CASE routed layer logits", bufs, flush=True)
    t = make(40, 128, 256, 16, BF)
    mine = torch.full((40, 16), 7.0, device=DEV)
    kept = {} if bufs else None
    if bufs:
        layer(t, 4, route=ROUTE, bufs=kept)
    r = layer(t, 4, route=ROUTE, logits=mine, bufs=kept)
    want = steps(t, 4, ROUTE)["logits"]
    assert r["logits"] is mine and torch.equal(mine, want)
    if bufs:  # and stay the caller's: a later call without it does not write there
        t["x"].mul_(2.0)
        after = layer(t, 4, route=ROUTE, bufs=kept)["logits"]
        assert after is not mine and torch.equal(mine, want) and not torch.equal(after, want)


def test_buffers_of_another_batch_are_refused():
    """Before anything is launched that would write past their ends."""
    print("CASE routed layer other batch", flush=True)
    t, kept = make(40, 128, 256, 16, BF), {}
    layer(t, 4, route=ROUTE, bufs=kept)
    for T in (39, 41):
        other = {**t, "x": make(T, 128, 256, 16, BF)["x"]}
        with pytest.raises(ValueError, match="logits"):
            layer(other, 4, route=ROUTE, bufs=kept)
        with pytest.raises(ValueError, match="logits"):
            layer(other, 4, route=ROUTE, logits=torch.empty((40, 16), device=DEV))
