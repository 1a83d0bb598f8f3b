"""A training step of a layer with group-routed and shared experts, all calls together: forward
through moe_layer with moe_route, a gated shared expert added to the routed ones' output,
dropout with the residual; backwards to the shared expert, the router and the tokens, against
float64 autograd on the same selection and mask.

Tolerance (fixed before any GPU run): fp32 throughout. A value is the result of at most four
chained products (the router's, two of an expert's, one of a gradient) of n <= 256 terms of
random sign, each off by n 2^-24 of its terms' sizes at most, and the sizes of n random terms are
sqrt(n) times their sum: 4 * 256 * 16 * 2^-24 = 1e-3 of the root mean square of a result would
never be passed; the errors too are random, so 1e-4 is asked for, as of fp32 layer outputs
elsewhere.
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
T, H, I, E, K = 48, 128, 256, 8, 2
P, SEED, OFFSET = 0.25, 99, 5


def near(got, want, what):
    got, want = got.double(), want.double()
    rms = float(want.pow(2).mean().sqrt())
    err = float((got - want).abs().max())
    assert err <= 1e-4 * rms, (what, err, rms)


def make():
    g = torch.Generator(device=DEV)
    g.manual_seed(5)

    def n(*shape):
        return torch.randn(shape, generator=g, device=DEV) / shape[-1] ** 0.5

    t = {"x": n(T, H) * H ** 0.5, "wr": n(E, H), "bias": 0.1 * n(1, E)[0], "wg": n(E, I, H), "wu": n(E, I, H), "wd": n(E, H, I),
         "sg": n(I, H), "su": n(I, H), "sd": n(H, I), "sb": n(1, I)[0], "dout": n(T, H) * H ** 0.5}
    t["rng"] = torch.tensor([SEED, OFFSET], device=DEV)
    return t


def forward(t, route, bufs, z, h):
    r = moe.moe_layer(t["x"], t["wr"], t["bias"], K, np.arange(E, dtype=np.int32), t["wg"], t["wu"], t["wd"], bufs=bufs, route=route)
    u = moe.moe_linear(t["x"], t["su"])
    moe.moe_linear(t["x"], t["sg"], bias=t["sb"], act="silu", mul=u, z=z, out=h)
    y = moe.moe_linear(h, t["sd"], residual=r["out"])
    return r, u, moe.moe_dropout_add(y, P, t["rng"], residual=t["x"])


def backward(t, route, r, u, z, h):
    dy = moe.moe_dropout_add(t["dout"], P, t["rng"])
    dh, dsd, _, _, _ = moe.moe_linear_backward(dy, h, t["sd"], need_dbias=False)
    dx, dsg, dsb, _, du = moe.moe_linear_backward(dh, t["x"], t["sg"], z=z, act="silu", mul=u)
    dx2, dsu, _, _, _ = moe.moe_linear_backward(du, t["x"], t["su"], need_dbias=False)
    dw, _ = moe.moe_combine_backward(dy, r["y_perm"], r["weights"], r["dest"], need_dy=False)
    kind = {n: route[n] for n in ("score", "norm", "scale")}
    dz = moe.moe_route_backward(r["logits"], r["ids"], dw, **kind)
    dx3, dwr, _, _ = moe.moe_router_grad(dz, t["x"], t["wr"])
    return {"sd": dsd, "sg": dsg, "sb": dsb, "su": dsu, "wr": dwr, "x": t["dout"] + dx + dx2 + dx3}


def reference(t, route, ids):
    """float64 on the same experts and mask; the routed experts are frozen and their input is
    taken as given (their gradient to x is not computed by the step)."""
    d = {n: v.double() for n, v in t.items() if n not in ("rng",)}
    leaf = {n: d[n].clone().requires_grad_() for n in ("x", "wr", "sg", "su", "sd", "sb")}
    x = leaf["x"]
    logits = x @ leaf["wr"].t()
    s = torch.sigmoid(logits) if route["score"] == "sigmoid" else torch.softmax(logits, 1)
    w = s.gather(1, ids.long())
    if route["norm"]:
        w = w / w.sum(1, keepdim=True)
    w = w * route["scale"]
    routed = torch.zeros_like(x)
    for j in range(K):
        e = ids[:, j].long()
        f = d["x"].unsqueeze(2)
        g, u = (d["wg"][e] @ f).squeeze(2), (d["wu"][e] @ f).squeeze(2)
        y = (d["wd"][e] @ (torch.nn.functional.silu(g) * u).unsqueeze(2)).squeeze(2)
        routed = routed + w[:, j:j + 1] * y
    h = torch.nn.functional.silu(x @ leaf["sg"].t() + leaf["sb"]) * (x @ leaf["su"].t())
    y = h @ leaf["sd"].t() + routed
    words = torch.from_numpy((O.dropout_words(T * H, SEED, OFFSET) >= np.uint64(int(P * 2 ** 32))).astype(np.float64)).to(DEV)
    out = y * words.view(T, H) / (1 - P) + x
    out.backward(d["dout"])
    return out.detach(), {n: v.grad for n, v in leaf.items()}


ROUTES = [{"score": "sigmoid", "n_group": 4, "topk_group": 2, "norm": True, "scale": 2.5},
          {"score": "softmax", "n_group": 1, "topk_group": 1, "norm": False, "scale": 1.0}]


@pytest.mark.parametrize("route", ROUTES)
def test_step(route):
    print("CASE layer step", route, flush=True)
    t, z, h = make(), torch.empty((T, I), device=DEV), torch.empty((T, I), device=DEV)
    bufs = {}
    for _ in range(2):  # the second time into the first one's buffers
        r, u, out = forward(t, route, bufs, z, h)
        ids, w = O.route(r["logits"].cpu().numpy(), K, bias=t["bias"].double().cpu().numpy(), **route)
        assert np.array_equal(r["ids"].cpu().numpy(), ids)
        grads = backward(t, route, r, u, z, h)
        want_out, want = reference(t, route, r["ids"])
        near(out, want_out, "out")
        for n in want:
            near(grads[n], want[n], n)


def test_step_in_a_graph_beside_an_eager_one():
    """The whole step captured and replayed, with the eager step on another stream between the
    replays; the mask of every replay is that of the state it finds."""
    print("CASE layer step graph", flush=True)
    route = ROUTES[0]
    t, z, h = make(), torch.empty((T, I), device=DEV), torch.empty((T, I), device=DEV)
    bufs = {}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        r, u, _ = forward(t, route, bufs, z, h)
        backward(t, route, r, u, z, h)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r, u, out = forward(t, route, bufs, z, h)
        grads = backward(t, route, r, u, z, h)
    z2, h2, bufs2 = torch.empty_like(z), torch.empty_like(h), {}
    for i in range(3):
        t["rng"][1] = OFFSET + 7 * i
        t["x"].mul_(1.0 + 0.1 * i)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            side.wait_stream(torch.cuda.current_stream())
            r2, u2, out2 = forward(t, route, bufs2, z2, h2)
            grads2 = backward(t, route, r2, u2, z2, h2)
        torch.cuda.synchronize()
        assert torch.equal(out, out2) and torch.equal(r["ids"], r2["ids"])
        for n in grads:
            assert torch.equal(grads[n], grads2[n]), n


def test_two_streams_at_once():
    """Calls with workspaces and streams of their own do not disturb each other."""
    print("CASE two streams", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    M, N, Kd = 300, 512, 4096
    x = torch.randn((M, Kd), generator=g, device=DEV).bfloat16()
    ws = [torch.randn((N, Kd), generator=g, device=DEV).bfloat16() for _ in range(2)]
    want = [moe.moe_linear(x, w) for w in ws]
    wants = [moe.moe_linear_backward(v, x, w)[:3] for v, w in zip(want, ws)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                y = moe.moe_linear(x, ws[i])
                got[i].append((y, moe.moe_linear_backward(y, x, ws[i])[:3]))
    torch.cuda.synchronize()
    for i in range(2):
        for y, grads in got[i]:
            assert torch.equal(y, want[i]) and all(torch.equal(a, b) for a, b in zip(grads, wants[i]))
