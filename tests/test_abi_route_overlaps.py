"""CPU tests of operands that share memory: what routing or dropout could answer wrongly is refused,
before any launch. A call whose sharing is allowed passes the checks; without a GPU its launch
then fails, which is another status."""
import ctypes

import pytest
import torch

import paper_2606_00735_amd as moe

INVALID = 1
AT = {n: 0x100000 * (i + 1) for i, n in enumerate(
    "logits bias mask ids gate dlogits x res rng out".split())}

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="allowed calls would launch on made-up addresses")


@pytest.fixture(scope="module")
def L():
    return moe.load_library()


def test_route(L):
    def route(without=(), **at):
        a = {**AT, **at, **{n: None for n in without}}
        return L.moe_route(a["logits"], a["bias"], a["mask"], 8, 16, 2, 0, 1, 1, 1, 1.0, a["ids"], a["gate"], None)

    assert route() != INVALID  # ids, weights: 64 bytes each; logits 512, bias 64, mask 8
    for out in ("ids", "gate"):
        for other, size in (("logits", 512), ("bias", 64), ("mask", 8)):
            assert route(**{out: AT[other]}) == INVALID and route(**{out: AT[other] - 60}) == INVALID, (out, other)
            assert route(**{out: AT[other] + size - 4}) == INVALID and route(**{out: AT[other] + size}) != INVALID, (out, other)
    assert route(ids=AT["gate"]) == INVALID and route(ids=AT["gate"] + 60) == INVALID and route(ids=AT["gate"] + 64) != INVALID
    assert route(["bias"], ids=AT["bias"]) != INVALID


def test_route_backward(L):
    def back(**at):
        a = {**AT, **at}
        return L.moe_route_backward(a["logits"], a["ids"], a["gate"], 8, 16, 2, 0, 1, 1.0, 0, a["dlogits"], None)

    assert back() != INVALID
    for other, size in (("logits", 512), ("ids", 64), ("gate", 64)):
        assert back(dlogits=AT[other]) == INVALID and back(dlogits=AT[other] - 496) == INVALID, other
        assert back(dlogits=AT[other] + size - 16) == INVALID and back(dlogits=AT[other] + size) != INVALID, other


def test_dropout(L):
    def drop(**at):
        a = {**AT, **at}
        return L.moe_dropout_add(a["x"], a["res"], 100, 0.5, a["rng"], 1, a["out"], None)

    assert drop() != INVALID
    for other in ("x", "res"):
        assert drop(out=AT[other]) != INVALID  # itself
        assert drop(out=AT[other] + 16) == INVALID and drop(out=AT[other] - 192) == INVALID, other
        assert drop(out=AT[other] + 208) != INVALID
    assert drop(rng=AT["out"]) == INVALID and drop(rng=AT["out"] + 192) == INVALID and drop(rng=AT["out"] + 200) != INVALID
    assert drop(x=AT["res"], out=AT["res"]) != INVALID
