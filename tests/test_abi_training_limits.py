"""CPU tests of the largest sizes that the training calls take: what lies beyond is
refused before a launch, what lies within passes the checks."""
import ctypes

import pytest

import paper_2606_00735_amd as moe

UNSUPPORTED = 2
FAKE = ctypes.c_void_p(0x10000)


@pytest.fixture(scope="module")
def L():
    return moe.load_library()


@pytest.mark.parametrize("T,E,k,seq,fits", [
    (2 ** 31 - 1, 4, 1, 0, False),    # 2^23 blocks of 256 tokens; token indices pass 2^31
    (2 ** 31 - 256, 4, 1, 0, True),   # one block fewer
    (2 ** 31 - 255, 4, 1, 0, False),
    (2 ** 23, 8, 2, 1, False),        # 2^23 groups: 2^32 threads of the loss
    (2 ** 23 - 1, 8, 2, 1, True),
    (2 ** 28 - 32, 32, 4, 0, True),
])
def test_balance_block_limit(L, T, E, k, seq, fits):
    n = ctypes.c_size_t(0)
    st = L.moe_balance_loss(None, None, None, T, E, k, seq, None, None, None, None, ctypes.byref(n), None)
    assert st == (0 if fits else UNSUPPORTED)
    if not fits:  # nothing is launched
        n = ctypes.c_size_t(1 << 40)
        assert L.moe_balance_loss(FAKE, FAKE, None, T, E, k, seq, FAKE, FAKE, FAKE, FAKE, ctypes.byref(n), None) == UNSUPPORTED
        assert L.moe_gate_backward(FAKE, FAKE, None, FAKE, FAKE, FAKE, None, None, T, E, k, seq, FAKE, None) == UNSUPPORTED
