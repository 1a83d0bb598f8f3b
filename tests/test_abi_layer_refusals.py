"""CPU tests of the refusals of routing, dense products and dropout, one reason at a time: every
operand has memory of its own, the unchanged call passes the checks (without a GPU its launch
then fails, which is another status), and each change alone is refused."""
import ctypes

import pytest
import torch

import paper_2606_00735_amd as moe

INVALID = 1
AT = {n: 0x100000 * (i + 1) for i, n in enumerate(
    "logits bias mask ids w dlogits dw x wt b mul res y z ws dy dz dmul dx dwt db rng out".split())}

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="allowed calls would launch on made-up addresses")


@pytest.fixture(scope="module")
def L():
    return moe.load_library()


def odd(name, by=4):
    return {name: AT[name] + by}


def route(L, T=4, E=16, k=2, score=0, G=4, g=2, scale=1.0, **at):
    a = {**AT, **at}
    return L.moe_route(a["logits"], a["bias"], a["mask"], T, E, k, score, G, g, 1, scale, a["ids"], a["w"], None)


def route_backward(L, T=4, E=16, k=2, score=0, scale=1.0, **at):
    a = {**AT, **at}
    return L.moe_route_backward(a["logits"], a["ids"], a["dw"], T, E, k, score, 1, scale, 0, a["dlogits"], None)


def linear(L, M=4, N=16, K=24, ld=0, act=2, dt=1, **at):
    a = {**AT, **at}
    n = ctypes.c_size_t(1 << 40)
    return L.moe_linear(a["x"], a["wt"], a["b"], a["mul"], a["res"], M, N, K, ld, act, dt, a["y"], a["z"], a["ws"], ctypes.byref(n), None)


def linear_backward(L, M=4, N=16, K=24, ld=0, act=2, dt=1, dwt_dt=1, **at):
    a = {**AT, **at}
    n = ctypes.c_size_t(1 << 40)
    return L.moe_linear_backward(a["dy"], a["x"], a["wt"], a["z"], a["mul"], M, N, K, ld, act, dt, a["dz"], a["dmul"], a["dx"], a["dwt"],
                                 dwt_dt, a["db"], a["ws"], ctypes.byref(n), None)


def dropout(L, n=10, p=0.5, dt=1, **at):
    a = {**AT, **at}
    return L.moe_dropout_add(a["x"], a["res"], n, p, a["rng"], dt, a["out"], None)


PLAIN = dict(mul=None, dmul=None, dz=None, z=None, act=0)  # dz is dy
ALLOWED = [(route, {}), (route, dict(bias=None, mask=None)), (route, odd("bias")), (route, odd("ids")), (route, odd("w")), (route, odd("mask", 1)),
           (route_backward, {}), (route_backward, odd("ids")), (route_backward, odd("dw")), (linear, {}), (linear, dict(b=None, mul=None, res=None, z=None)),
           (linear, dict(ld=32)), (linear, dict(dt=0, ld=28)), (linear_backward, {}), (linear_backward, PLAIN), (linear_backward, dict(dmul=None)),
           (linear_backward, dict(dx=None, wt=None)), (linear_backward, dict(dwt=None, x=None)), (linear_backward, dict(db=None)),
           (linear_backward, dict(dt=0, dwt_dt=0)), (linear_backward, dict(dwt_dt=0)), (dropout, {}), (dropout, dict(res=None)), (dropout, dict(p=0.0)),
           (dropout, odd("rng", 8))]
REFUSED = ([(route, c) for c in [dict(T=-1), dict(E=0), dict(E=257), dict(k=0), dict(k=17, E=64), dict(k=9), dict(score=2), dict(G=0), dict(G=5),
                                 dict(G=32), dict(g=0), dict(g=5), dict(scale=1e39), dict(logits=None), dict(ids=None), dict(w=None), odd("logits"),
                                 odd("ids", 2), odd("w", 2), odd("bias", 2)]]
           + [(route_backward, c) for c in [dict(T=-1), dict(E=300), dict(k=17, E=64), dict(k=3, E=2), dict(score=3), dict(scale=-1e39), dict(logits=None),
                                            dict(ids=None), dict(dw=None), dict(dlogits=None), odd("logits"), odd("dlogits"), odd("dw", 2),
                                            odd("ids", 2)]]
           + [(linear, c) for c in [dict(M=-1), dict(N=0), dict(N=12), dict(K=20), dict(dt=2), dict(act=4), dict(act=-1), dict(ld=16), dict(ld=28),
                                    dict(ld=(1 << 20) + 8), dict(x=None), dict(wt=None), dict(y=None)] + [odd(n) for n in "x wt b mul res y z ws".split()]]
           + [(linear_backward, c) for c in [dict(M=-1), dict(N=4), dict(K=9), dict(act=9), dict(dt=0), dict(dwt_dt=2), dict(dy=None), dict(x=None),
                                             dict(wt=None), dict(z=None), dict(z=None, dmul=None), dict(dz=None), dict(mul=None),
                                             dict(act=0, z=None), {**PLAIN, "dmul": AT["dmul"]}]
              + [odd(n) for n in "dy x wt z mul dz dmul dx dwt db ws".split()]]
           + [(dropout, c) for c in [dict(n=-1), dict(p=1.0), dict(p=-0.1), dict(p=float("nan")), dict(dt=3), dict(x=None), dict(rng=None), dict(out=None),
                                     odd("x"), odd("res"), odd("out"), odd("rng")]])


@pytest.mark.parametrize("call,change", ALLOWED)
def test_allowed(L, call, change):
    assert call(L, **change) != INVALID


@pytest.mark.parametrize("call,change", REFUSED)
def test_refused(L, call, change):
    assert call(L, **change) == INVALID
