"""CPU tests of the argument checks of the MXFP4 entry points: no call reaches a launch."""
import ctypes

import pytest

import paper_2606_00735_amd as moe

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
FAKE, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10004)
NULL = ctypes.c_void_p(None)


@pytest.fixture(scope="module")
def L():
    return moe.load_library()


@pytest.mark.parametrize("x,dt,batch,rows,K,ld,rc,codes,want", [
    (FAKE, 7, 1, 4, 256, 0, None, FAKE, INVALID),        # dtype
    (FAKE, 1, 1, -1, 256, 0, None, FAKE, INVALID),
    (FAKE, 1, 1, 4, 0, 0, None, FAKE, INVALID),
    (FAKE, 1, 1, 4, 48, 0, None, FAKE, UNSUPPORTED),     # K % 32
    (FAKE, 1, 1, 4, (1 << 20) + 32, 0, None, FAKE, UNSUPPORTED),
    (FAKE, 1, 2 ** 30, 2 ** 30, 256, 0, None, FAKE, UNSUPPORTED),
    (FAKE, 1, 1, 4, 256, 64, None, FAKE, INVALID),       # rows shorter than their codes
    (FAKE, 1, 1, 4, 256, 136, None, FAKE, INVALID),      # no multiple of 16
    (FAKE, 1, 2, 4, 256, 0, FAKE, FAKE, INVALID),        # row_count of a batch
    (NULL, 1, 1, 4, 256, 0, None, FAKE, INVALID),
    (ODD, 1, 1, 4, 256, 0, None, FAKE, INVALID),
    (FAKE, 1, 1, 4, 256, 0, None, ODD, INVALID),
    (NULL, 1, 1, 0, 256, 0, None, NULL, 0),              # no rows
])
def test_quantize_checks(L, x, dt, batch, rows, K, ld, rc, codes, want):
    assert L.moe_mx4_quantize(x, dt, batch, rows, K, ld, rc, codes, FAKE, None) == want
    if rc is None and dt == 1:
        assert L.moe_mx4_dequantize(codes, FAKE, batch, rows, K, ld, x, None) == want


def _ffn(L, src=None, T=0, k=0, E_local=2, H=256, I=128, ldg=0, ldd=0, M=16, y=FAKE, ws=FAKE, n=1 << 40, x=FAKE):
    n = ctypes.c_size_t(n)
    st = L.moe_grouped_swiglu_ffn_mx4(x, FAKE, src, T, k, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, E_local, H, I, ldg,
                                      ldd, M, y, ws, ctypes.byref(n), None)
    return st, n.value


@pytest.mark.parametrize("args,want", [
    (dict(E_local=-1), INVALID), (dict(E_local=257), UNSUPPORTED), (dict(H=200), UNSUPPORTED), (dict(I=64), UNSUPPORTED),
    (dict(M=-1), INVALID), (dict(ldg=100), INVALID), (dict(ldd=8), INVALID),
    (dict(src=FAKE, T=0, k=2), INVALID), (dict(src=FAKE, T=4, k=0), INVALID), (dict(src=FAKE, T=4, k=17), INVALID),
    (dict(src=ODD, T=2 ** 25, k=1), UNSUPPORTED), (dict(src=ctypes.c_void_p(0x10002), T=4, k=1), INVALID),
    (dict(n=100), WORKSPACE), (dict(y=NULL), INVALID), (dict(x=ODD), INVALID), (dict(ws=ODD), INVALID),
    (dict(E_local=0), 0), (dict(M=0), 0),
])
def test_ffn_checks(L, args, want):
    assert _ffn(L, **args)[0] == want


def test_ffn_workspace_query(L):
    st, n = _ffn(L, ws=NULL, n=0)
    assert st == 0 and n >= 16384 + 16 * 128 + 16 * 8
    assert _ffn(L, n=n - 1)[0] == WORKSPACE


@pytest.mark.parametrize("N,K,ldb,M,c,want", [
    (100, 256, 0, 4, FAKE, UNSUPPORTED), (128, 96, 0, 4, FAKE, UNSUPPORTED), (128, 256, 120, 4, FAKE, INVALID),
    (128, 256, 0, -1, FAKE, INVALID), (128, 256, 0, 4, NULL, INVALID), (128, 256, 0, 0, NULL, 0),
])
def test_gemm_checks(L, N, K, ldb, M, c, want):
    assert L.moe_grouped_gemm_mx4(FAKE, FAKE, FAKE, FAKE, FAKE, 1, N, K, ldb, M, c, None) == want


# ---------------------------------------------------------------- the router's training step
def _loss(L, T=64, E=8, k=2, seq=0, z=FAKE, ids=FAKE, mask=NULL, loss=FAKE, counts=FAKE, live=FAKE, ws=FAKE, n=1 << 40):
    n = ctypes.c_size_t(n)
    return L.moe_balance_loss(z, ids, mask, T, E, k, seq, loss, counts, live, ws, ctypes.byref(n), None), n.value


@pytest.mark.parametrize("args,want", [
    (dict(T=-1), INVALID), (dict(E=0), INVALID), (dict(E=257), INVALID), (dict(k=0), INVALID), (dict(k=9), INVALID),
    (dict(E=32, k=17), INVALID), (dict(seq=-1), INVALID), (dict(seq=5), INVALID), (dict(T=2 ** 31 - 1, k=2), UNSUPPORTED),
    (dict(T=2 ** 24, seq=1), UNSUPPORTED), (dict(n=16), WORKSPACE), (dict(z=NULL), INVALID), (dict(z=ODD), INVALID),
    (dict(ids=ctypes.c_void_p(2)), INVALID), (dict(loss=NULL), INVALID), (dict(counts=NULL), INVALID),
    (dict(live=NULL), INVALID), (dict(ws=ODD), INVALID), (dict(T=0, loss=NULL), INVALID),
])
def test_balance_loss_checks(L, args, want):
    assert _loss(L, **args)[0] == want


def test_balance_loss_workspace_query(L):
    for T, E, k, seq in ((0, 8, 2, 0), (64, 8, 2, 0), (16384, 256, 8, 4096), (5000, 60, 4, 1)):
        st, n = _loss(L, T=T, E=E, k=k, seq=seq, ws=NULL)
        assert st == 0 and n >= 256 and n % 256 == 0
        assert _loss(L, T=T, E=E, k=k, seq=seq, n=n - 1)[0] == WORKSPACE


def _gate(L, T=64, E=8, k=2, seq=0, z=FAKE, w=NULL, dw=NULL, dz=FAKE, live=FAKE):
    return L.moe_gate_backward(z, FAKE, NULL, FAKE, live, FAKE, w, dw, T, E, k, seq, dz, None)


@pytest.mark.parametrize("args,want", [
    (dict(T=-1), INVALID), (dict(k=9), INVALID), (dict(seq=7), INVALID), (dict(w=FAKE), INVALID), (dict(dw=FAKE), INVALID),
    (dict(z=NULL), INVALID), (dict(z=ODD), INVALID), (dict(dz=NULL), INVALID), (dict(dz=ODD), INVALID),
    (dict(live=NULL), INVALID), (dict(T=2 ** 24, seq=1), UNSUPPORTED), (dict(T=0, z=NULL, dz=NULL), 0),
])
def test_gate_backward_checks(L, args, want):
    assert _gate(L, **args) == want


def _combine(L, T=4, k=2, H=64, M=8, dt=1, do=FAKE, y=FAKE, w=FAKE, dw=FAKE, dy=FAKE):
    return L.moe_combine_backward(do, y, w, FAKE, T, k, H, M, dt, dw, dy, None)


@pytest.mark.parametrize("args,want", [
    (dict(T=-1), INVALID), (dict(k=0), INVALID), (dict(k=17), INVALID), (dict(H=0), INVALID), (dict(H=12), INVALID),
    (dict(H=6, dt=0), INVALID), (dict(M=-1), INVALID), (dict(dt=5), INVALID), (dict(T=2 ** 30, k=4), UNSUPPORTED),
    (dict(do=NULL), INVALID), (dict(y=NULL), INVALID), (dict(w=NULL), INVALID), (dict(dw=NULL), INVALID),
    (dict(do=ODD), INVALID), (dict(y=ODD), INVALID), (dict(dy=ODD), INVALID), (dict(T=0, do=NULL), 0),
])
def test_combine_backward_checks(L, args, want):
    assert _combine(L, **args) == want


def _router(L, T=4, E=8, H=64, dt=1, dz=FAKE, x=FAKE, w=FAKE, dx=FAKE, dw=FAKE, db=FAKE, ws=FAKE, n=1 << 40):
    n = ctypes.c_size_t(n)
    return L.moe_router_grad(dz, x, w, T, E, H, dt, dx, dw, db, ws, ctypes.byref(n), None), n.value


@pytest.mark.parametrize("args,want", [
    (dict(T=-1), INVALID), (dict(E=0), INVALID), (dict(E=257), INVALID), (dict(H=0), INVALID), (dict(H=60), INVALID),
    (dict(H=72), UNSUPPORTED), (dict(H=(1 << 20) + 64), UNSUPPORTED), (dict(dt=3), INVALID), (dict(n=16), WORKSPACE),
    (dict(dz=NULL), INVALID), (dict(x=NULL), INVALID), (dict(w=NULL), INVALID), (dict(dw=NULL), INVALID),
    (dict(db=NULL), INVALID), (dict(dz=ODD), INVALID), (dict(x=ODD), INVALID), (dict(dx=ODD), INVALID),
    (dict(dw=ODD), INVALID), (dict(ws=ODD), INVALID),
])
def test_router_grad_checks(L, args, want):
    assert _router(L, **args)[0] == want


def test_router_grad_workspace_query(L):
    st, n = _router(L, T=16384, E=256, H=7168, ws=NULL)
    assert st == 0 and n >= 2 * 256 * 7168 * 4  # at least two ranges of tokens
    assert _router(L, T=16384, E=256, H=7168, n=n - 1)[0] == WORKSPACE
    st, n = _router(L, T=8, ws=NULL)
    assert st == 0 and n == 256
