"""CPU tests of operands that share memory: what a dense product could answer wrongly is refused,
before any launch. A call whose sharing is allowed passes the checks; without a GPU its launch
then fails, which is another status."""
import ctypes

import pytest
import torch

import paper_2606_00735_amd as moe

INVALID = 1
M, N, K = 4, 16, 16  # bf16 [M, N], [M, K]: 128 bytes, [N, K]: 512
AT = {n: 0x100000 * (i + 1) for i, n in enumerate(
    "x w bias mul res y z ws dy dz dmul dx dw db".split())}

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="allowed calls would launch on made-up addresses")


@pytest.fixture(scope="module")
def L():
    return moe.load_library()


def linear(L, without=(), m=M, **at):
    a = {**AT, **at, **{n: None for n in without}}
    n = ctypes.c_size_t(1 << 40)
    return L.moe_linear(a["x"], a["w"], a["bias"], a["mul"], a["res"], m, N, K, 0, 1, 1, a["y"], a["z"], a["ws"], ctypes.byref(n),
                        None)


def test_linear(L):
    ok = linear(L)
    assert ok != INVALID
    for out in ("y", "z"):
        for other in ("x", "w", "bias"):
            assert linear(L, **{out: AT[other]}) == INVALID, (out, other)
            assert linear(L, **{out: AT[other] + 16}) == INVALID, (out, other)  # in part
    assert linear(L, y=AT["z"]) == INVALID and linear(L, y=AT["z"] + 112) == INVALID
    # the last 16 bytes of w [16, 16], and the first after it
    assert linear(L, y=AT["w"] + 496) == INVALID and linear(L, y=AT["w"] + 512) != INVALID
    assert linear(L, y=AT["x"] - 112) == INVALID and linear(L, y=AT["x"] - 128) != INVALID
    for other in ("mul", "res"):
        assert linear(L, y=AT[other]) != INVALID  # itself, element by element
        assert linear(L, y=AT[other] + 16) == INVALID and linear(L, y=AT[other] - 16) == INVALID
        assert linear(L, z=AT[other]) == INVALID and linear(L, z=AT[other] + 64) == INVALID
    assert linear(L, mul=AT["res"], y=AT["res"]) != INVALID
    # what is not there shares nothing
    assert linear(L, ["bias"], y=AT["bias"]) != INVALID and linear(L, ["z"], y=AT["z"]) != INVALID
    assert linear(L, m=0, y=AT["x"]) == 0
    for other in ("x", "w", "bias", "mul", "res", "y", "z"):  # 256 bytes of workspace
        assert linear(L, ws=AT[other]) == INVALID and linear(L, ws=AT[other] - 240) == INVALID, other
        assert linear(L, ws=AT[other] - 256) != INVALID, other


def backward(L, without=(), act=1, m=M, dwt=1, **at):
    a = {**AT, **at, **{n: None for n in without}}
    n = ctypes.c_size_t(1 << 40)
    return L.moe_linear_backward(a["dy"], a["x"], a["w"], a["z"], a["mul"], m, N, K, 0, act, 1, a["dz"], a["dmul"], a["dx"], a["dw"], dwt,
                                 a["db"], a["ws"], ctypes.byref(n), None)


PLAIN = ["mul", "dmul", "dz"]


def test_linear_backward(L):
    assert backward(L) != INVALID and backward(L, PLAIN, act=0) != INVALID
    # the pass that writes dz and dmul comes before the products that read x and w
    for out in ("dz", "dmul"):
        for other in ("x", "w"):
            assert backward(L, **{out: AT[other]}) == INVALID, (out, other)
            assert backward(L, **{out: AT[other] + 64}) == INVALID, (out, other)
        assert backward(L, **{out: AT["w"] + 512}) != INVALID
    # not where that product is not asked for
    assert backward(L, ["dw"], dz=AT["x"]) != INVALID and backward(L, ["dx"], dz=AT["w"]) != INVALID
    for other in ("z", "mul"):
        for out in ("dz", "dmul"):
            assert backward(L, **{out: AT[other]}) == INVALID and backward(L, **{out: AT[other] + 16}) == INVALID, (out, other)
    assert backward(L, dz=AT["dy"]) != INVALID  # element by element
    assert backward(L, dz=AT["dy"] + 16) == INVALID
    assert backward(L, dmul=AT["dy"]) == INVALID and backward(L, dmul=AT["dy"] + 16) == INVALID
    # the bias' sums share nothing
    for other in ("dy", "x", "w", "z", "mul", "dz", "dmul", "dx", "dw"):
        assert backward(L, db=AT[other]) == INVALID, other
        assert backward(L, db=AT[other] + 16) == INVALID, other
    assert backward(L, PLAIN, act=0, db=AT["dy"]) == INVALID
    # the products' outputs
    for out in ("dx", "dw"):
        for other in ("dy", "x", "w", "dz", "dmul"):
            assert backward(L, **{out: AT[other]}) == INVALID and backward(L, **{out: AT[other] + 32}) == INVALID, (out, other)
        # read by the pass before them alone
        assert backward(L, **{out: AT["z"]}) != INVALID and backward(L, **{out: AT["mul"]}) != INVALID
    assert backward(L, dx=AT["dw"] + 496) == INVALID and backward(L, dx=AT["dw"] + 512) != INVALID
    assert backward(L, dx=AT["dw"] + 1008, dwt=0) == INVALID and backward(L, dx=AT["dw"] + 1024, dwt=0) != INVALID
    assert backward(L, dz=AT["dmul"] + 16) == INVALID
    for other in ("dy", "x", "w", "z", "mul", "dz", "dmul", "dx", "dw", "db"):
        assert backward(L, ws=AT[other]) == INVALID and backward(L, ws=AT[other] - 240) == INVALID, other
    # no rows: dw and dbias are written all the same
    assert backward(L, m=0, db=AT["dw"] + 64) == INVALID
