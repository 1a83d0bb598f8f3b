"""CPU tests of the argument checks of routing, dense products and dropout: no call reaches
a launch."""
import ctypes
import math

import pytest
import torch

import paper_2606_00735_amd as moe

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
FAKE, FAKE2, FAKE3 = (ctypes.c_void_p(v) for v in (0x10000, 0x20000, 0x30000))
ODD, ODD4 = ctypes.c_void_p(0x10004), ctypes.c_void_p(0x10002)
NULL = ctypes.c_void_p(None)


@pytest.fixture(scope="module")
def L():
    return moe.load_library()


def route(L, z=FAKE, bias=None, mask=None, T=4, E=16, k=2, score=0, G=4, g=2, norm=1, scale=1.0, ids=FAKE, w=FAKE):
    return L.moe_route(z, bias, mask, T, E, k, score, G, g, norm, scale, ids, w, None)


@pytest.mark.parametrize("args,want", [
    (dict(T=-1), INVALID), (dict(E=0), INVALID), (dict(E=257), INVALID), (dict(k=0), INVALID), (dict(k=17, E=32), INVALID),
    (dict(score=2), INVALID), (dict(score=-1), INVALID), (dict(G=0), INVALID), (dict(G=5), INVALID), (dict(G=32), INVALID),
    (dict(g=0), INVALID), (dict(g=5), INVALID),
    (dict(k=9), INVALID),                      # two groups of four hold eight experts
    (dict(scale=math.inf), INVALID), (dict(scale=math.nan), INVALID), (dict(T=2 ** 30, k=2), UNSUPPORTED),
    (dict(z=NULL), INVALID), (dict(ids=NULL), INVALID), (dict(w=NULL), INVALID), (dict(z=ODD), INVALID),
    (dict(ids=ODD4), INVALID), (dict(w=ODD4), INVALID), (dict(bias=ODD4), INVALID),
    (dict(T=0, z=NULL, ids=NULL, w=NULL), 0),
    (dict(scale=1e39), INVALID), (dict(scale=-1e39), INVALID),  # not finite in fp32
])
def test_route_checks(L, args, want):
    assert route(L, **args) == want


def route_backward(L, z=FAKE, ids=FAKE, dw=FAKE, T=4, E=16, k=2, score=0, norm=1, scale=1.0, acc=0, dz=FAKE2):
    return L.moe_route_backward(z, ids, dw, T, E, k, score, norm, scale, acc, dz, None)


@pytest.mark.parametrize("args,want", [
    (dict(T=-1), INVALID), (dict(E=300), INVALID), (dict(k=17), INVALID), (dict(score=3), INVALID),
    (dict(scale=math.inf), INVALID), (dict(z=NULL), INVALID), (dict(ids=NULL), INVALID), (dict(dw=NULL), INVALID),
    (dict(dz=NULL), INVALID), (dict(dz=FAKE), INVALID), (dict(z=ODD), INVALID), (dict(dz=ODD), INVALID),
    (dict(dw=ODD4), INVALID), (dict(T=0, z=NULL, ids=NULL, dw=NULL, dz=NULL), 0),
    (dict(scale=1e39), INVALID), (dict(dw=FAKE2, E=2), INVALID),
])
def test_route_backward_checks(L, args, want):
    assert route_backward(L, **args) == want


def linear(L, x=FAKE, w=FAKE2, bias=None, mul=None, res=None, M=4, N=16, K=24, ld=0, act=0, dt=1, y=FAKE3, z=None, ws=FAKE,
           n=1 << 40):
    n = ctypes.c_size_t(n)
    return L.moe_linear(x, w, bias, mul, res, M, N, K, ld, act, dt, y, z, ws, ctypes.byref(n), None), n.value


@pytest.mark.parametrize("args,want", [
    (dict(M=-1), INVALID), (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(N=12), INVALID), (dict(K=20), INVALID),
    (dict(dt=2), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID), (dict(ld=16), INVALID), (dict(ld=28), INVALID),
    (dict(ld=(1 << 20) + 8), INVALID), (dict(N=(1 << 20) + 8), UNSUPPORTED), (dict(K=(1 << 20) + 8), UNSUPPORTED),
    (dict(M=(1 << 28) + 1), UNSUPPORTED), (dict(M=1 << 28, N=512), UNSUPPORTED), (dict(M=1 << 28, K=512), UNSUPPORTED),
    (dict(M=1 << 28, N=128, K=8, dt=0), UNSUPPORTED), (dict(N=1 << 19, K=1 << 18), UNSUPPORTED),
    (dict(n=100), WORKSPACE), (dict(x=NULL), INVALID), (dict(w=NULL), INVALID), (dict(y=NULL), INVALID),
    (dict(y=FAKE), INVALID), (dict(y=FAKE2), INVALID), (dict(z=FAKE3), INVALID), (dict(z=FAKE), INVALID),
    (dict(x=ODD), INVALID), (dict(w=ODD), INVALID), (dict(y=ODD), INVALID), (dict(z=ODD), INVALID),
    (dict(bias=ODD), INVALID), (dict(mul=ODD), INVALID), (dict(res=ODD), INVALID), (dict(ws=ODD), INVALID),
    (dict(M=0, x=NULL, w=NULL, y=NULL), 0),
])
def test_linear_checks(L, args, want):
    assert linear(L, **args)[0] == want


def backward(L, dy=FAKE, x=FAKE2, w=FAKE3, z=None, mul=None, M=4, N=16, K=24, ld=0, act=0, dt=1, dz=None, dmul=None,
             dx=ctypes.c_void_p(0x40000), dw=ctypes.c_void_p(0x50000), dwt=1, db=FAKE, ws=FAKE, n=1 << 40):
    n = ctypes.c_size_t(n)
    return L.moe_linear_backward(dy, x, w, z, mul, M, N, K, ld, act, dt, dz, dmul, dx, dw, dwt, db, ws, ctypes.byref(n),
                                 None), n.value


A, B, C, D = (ctypes.c_void_p(0x60000 + 0x10000 * i) for i in range(4))


@pytest.mark.parametrize("args,want", [
    (dict(M=-1), INVALID), (dict(N=4), INVALID), (dict(K=9), INVALID), (dict(act=9), INVALID), (dict(dt=0, dwt=1), INVALID),
    (dict(dwt=2), INVALID), (dict(M=1 << 29), UNSUPPORTED), (dict(n=10), WORKSPACE), (dict(dy=NULL), INVALID),
    (dict(x=NULL), INVALID), (dict(w=NULL), INVALID),
    (dict(act=1), INVALID),                              # no z, no dz
    (dict(act=1, z=A), INVALID), (dict(act=1, dz=B), INVALID),
    (dict(mul=A), INVALID),                              # no dz
    (dict(mul=A, dz=B, dmul=C), INVALID),                # no z for dmul
    (dict(dmul=C), INVALID),                             # no mul
    (dict(mul=A, dz=B, dmul=B, z=D), INVALID), (dict(mul=A, dz=B, dmul=A, z=D), INVALID),
    (dict(mul=A, dz=B, dmul=FAKE, z=D), INVALID), (dict(act=2, z=A, dz=A), INVALID), (dict(mul=A, dz=A), INVALID),
    (dict(dx=FAKE), INVALID), (dict(dx=FAKE3), INVALID), (dict(dw=FAKE2), INVALID), (dict(act=2, z=A, dz=B, dx=B), INVALID),
    (dict(dy=ODD), INVALID), (dict(x=ODD), INVALID), (dict(w=ODD), INVALID), (dict(dx=ODD), INVALID), (dict(dw=ODD), INVALID),
    (dict(dw=ctypes.c_void_p(0x40000)), INVALID), (dict(db=ctypes.c_void_p(0x50000)), INVALID),  # one output twice
    (dict(mul=A, dz=B, dmul=ctypes.c_void_p(0x40000), z=D), INVALID),
    (dict(db=ODD), INVALID), (dict(ws=ODD), INVALID), (dict(act=2, z=ODD, dz=B), INVALID), (dict(act=2, z=A, dz=ODD), INVALID),
])
def test_linear_backward_checks(L, args, want):
    assert backward(L, **args)[0] == want


@pytest.mark.parametrize("M,N,K", [(0, 8, 8), (1, 8, 8), (1, 7168, 2048), (16384, 2048, 7168), (1 << 28, 256, 8)])
@pytest.mark.parametrize("dt", [0, 1])
def test_linear_workspace_queries(L, M, N, K, dt):
    if dt == 0 and M == 1 << 28:
        M = 1 << 26
    st, n = linear(L, M=M, N=N, K=K, dt=dt, ws=NULL, n=0)
    assert st == 0 and 0 < n <= (64 << 20)
    st, n = backward(L, M=M, N=N, K=K, dt=dt, dwt=dt, ws=NULL, n=0)
    assert st == 0 and 0 < n <= (128 << 20)


def dropout(L, x=FAKE, res=None, n=10, p=0.5, rng=FAKE2, dt=1, out=FAKE3):
    return L.moe_dropout_add(x, res, n, p, rng, dt, out, None)


@pytest.mark.parametrize("args,want", [
    (dict(n=-1), INVALID), (dict(n=(1 << 40) + 1), UNSUPPORTED), (dict(p=1.0), INVALID), (dict(p=-0.1), INVALID),
    (dict(p=math.nan), INVALID), (dict(dt=3), INVALID), (dict(x=NULL), INVALID), (dict(rng=NULL), INVALID),
    (dict(out=NULL), INVALID), (dict(x=ODD), INVALID), (dict(res=ODD), INVALID), (dict(out=ODD), INVALID),
    (dict(rng=ODD), INVALID), (dict(n=0, x=NULL, rng=NULL, out=NULL), 0),
])
def test_dropout_checks(L, args, want):
    assert dropout(L, **args) == want


def test_python_wrappers_refuse_cpu_tensors_and_wrong_names(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    x = torch.zeros(4, 16)
    with pytest.raises(ValueError, match="GPU"):
        moe.moe_route(x, 2)
    with pytest.raises(ValueError, match="GPU"):
        moe.moe_route_backward(x, torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, 2))
    with pytest.raises(ValueError, match="GPU"):
        moe.moe_linear(x, torch.zeros(8, 16))
    with pytest.raises(ValueError, match="GPU"):
        moe.moe_linear_backward(torch.zeros(4, 8), x, torch.zeros(8, 16))
    with pytest.raises(ValueError, match="GPU"):
        moe.moe_dropout_add(x, 0.1, torch.zeros(2, dtype=torch.int64))
    with pytest.raises(ValueError, match="score"):
        moe.moe_route(x, 2, score="tanh")
    with pytest.raises(ValueError, match="act"):
        moe.moe_linear(x, torch.zeros(8, 16), act="tanh")
    with pytest.raises(ValueError, match="dw_dtype"):
        moe.moe_linear_backward(torch.zeros(4, 8), x, torch.zeros(8, 16), dw_dtype=torch.float16)
    with pytest.raises(ValueError, match="accumulate"):
        moe.moe_route_backward(x, torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, 2), accumulate=True)
    with pytest.raises(TypeError):
        moe.moe_linear([1.0], torch.zeros(8, 16))
    with pytest.raises(ValueError, match="two dimensions"):
        moe.moe_linear(torch.zeros(2, 4, 16), torch.zeros(8, 16))
    assert [moe.dropout_counters(n) for n in (0, 1, 4, 5)] == [0, 1, 1, 2]
