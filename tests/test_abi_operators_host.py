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
