"""CPU tests of the dense products' workspaces: the size that a query names for M rows serves
every call of at most M rows, so a program sizes one buffer for its largest batch."""
import ctypes
import random

import pytest

import paper_2606_00735_amd as moe

INVALID, WORKSPACE = 1, 3
AT = 0x100000


@pytest.fixture(scope="module")
def L():
    return moe.load_library()


def forward(L, M, N, K, dt, ws, n):
    n = ctypes.c_size_t(n)
    # no x: a call whose workspace is large enough goes on to refuse that
    return L.moe_linear(None, AT, None, None, None, M, N, K, 0, 0, dt, 2 * AT, None, ws, ctypes.byref(n), None), n.value


def backward(L, M, N, K, dt, ws, n):
    n = ctypes.c_size_t(n)
    return L.moe_linear_backward(None, AT, AT, None, None, M, N, K, 0, 0, dt, None, None, 2 * AT, 3 * AT, dt, 4 * AT, ws, ctypes.byref(n),
                                 None), n.value


SIZES = [(4096, 14336), (14336, 4096), (2048, 7168), (7168, 2048), (2048, 768), (1336, 1000), (8, 8), (72, 16384), (16384, 72), (1000, 1336),
         (128, 128)]


@pytest.mark.parametrize("call", [forward, backward])
@pytest.mark.parametrize("dt", [0, 1])
def test_a_size_serves_fewer_rows(L, call, dt):
    r = random.Random(5)
    sizes = SIZES + [(8 * r.randint(1, 1500), 8 * r.randint(1, 1500)) for _ in range(20)]
    rows = sorted({1, 2, 8, 9, 32, 33, 64, 100, 255, 256, 300, 512, 768, 769, 1000, 1024, 1025, 1500, 2000, 2422, 4000, 8192, 16384,
                   *(r.randint(1, 20000) for _ in range(40))})
    for N, K in sizes:
        last = 0
        for i, M in enumerate(rows):
            st, n = call(L, M, N, K, dt, None, 0)
            assert st == 0 and n >= last, (M, N, K)
            last = n
            for m in rows[:i + 1]:
                assert call(L, m, N, K, dt, AT, n)[0] == INVALID, (m, M, N, K)
        assert call(L, rows[-1], N, K, dt, AT, 255)[0] == WORKSPACE


def test_sizes_stay_small(L):
    """Partial sums are 64 MiB at most; products that no rows would split need none."""
    assert forward(L, 16384, 14336, 4096, 1, None, 0)[1] <= 64 << 20
    assert forward(L, 16384, 4096, 448, 1, None, 0)[1] == 256
    assert forward(L, 1, 7168, 2048, 1, None, 0)[1] <= 1 << 20
    assert forward(L, 16384, 4096, 4096, 0, None, 0)[1] == 256
    assert backward(L, 8192, 7168, 2048, 1, None, 0)[1] <= 68 << 20
