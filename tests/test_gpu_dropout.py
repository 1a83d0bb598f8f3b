"""GPU tests of dropout with a residual against the oracle: masks exactly, values to the
roundings of an fp32 product (2^-24), a sum (2^-24) and the result (2^-8 in bf16)."""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import layer_oracle as O

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


def banner(*a):
    print("CASE", *a, flush=True)


def rng(seed, offset):
    wrap = lambda v: v - (1 << 64) if v >= 1 << 63 else v  # noqa: E731
    return torch.tensor([wrap(seed), wrap(offset)], dtype=torch.int64, device=DEV)


@pytest.mark.parametrize("n", [1, 3, 4, 5, 7, 8, 9, 255, 1024, 2049, 4099, 12345])
@pytest.mark.parametrize("dtype", [BF, torch.float32])
@pytest.mark.parametrize("res", [False, True])
def test_values(n, dtype, res):
    banner("dropout", n, dtype, res)
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    x = torch.randn(n, generator=g, device=DEV).to(dtype)
    r = torch.randn(n, generator=g, device=DEV).to(dtype) if res else None
    for p, seed, offset in ((0.1, 1234567890123456789, 5), (0.5, (1 << 64) - 3, (1 << 32) - 2), (0.9, 0, (1 << 64) - 1),
                            (0.0, 7, 7), (1 - 2.0 ** -40, 8, 8)):
        buf = torch.full((n + 64,), 7.0, device=DEV, dtype=dtype)
        out = buf[32:32 + n]
        y = moe.moe_dropout_add(x, p, rng(seed, offset), residual=r, out=out)
        assert (buf[:32] == 7).all() and (buf[32 + n:] == 7).all()
        xd, rd = x.double().cpu().numpy(), None if r is None else r.double().cpu().numpy()
        want = O.dropout_add(xd, p, seed, offset, rd)
        dropped = O.dropout_words(n, seed, offset) < np.uint64(int(p * 4294967296.0))
        got = y.double().cpu().numpy()
        base = np.zeros(n) if rd is None else rd
        assert np.array_equal(got[dropped], base[dropped])
        size = np.abs(want - base) + np.abs(want)
        tol = 2.0 ** -23 * size + (2.0 ** -8 if dtype == BF else 2.0 ** -24) * np.abs(want)
        assert np.all(np.abs(got - want) <= tol)


def test_dropped_values_are_not_read_into_the_result():
    banner("dropout NaN")
    n = 4096
    words = O.dropout_words(n, 3, 9)
    drop = torch.from_numpy(words < np.uint64(1 << 31)).to(DEV)
    x = torch.where(drop, torch.tensor(float("nan"), device=DEV), torch.ones(n, device=DEV))
    y = moe.moe_dropout_add(x, 0.5, rng(3, 9))
    assert torch.equal(y, torch.where(drop, 0.0, 2.0))


def test_in_place_and_gradient():
    banner("dropout in place")
    x, r = torch.randn((33, 130), device=DEV).to(BF), torch.randn((33, 130), device=DEV).to(BF)
    s = rng(11, 1)
    want = moe.moe_dropout_add(x, 0.3, s, residual=r)
    a = x.clone()
    assert moe.moe_dropout_add(a, 0.3, s, residual=r, out=a) is a and torch.equal(a, want)
    b = r.clone()
    assert torch.equal(moe.moe_dropout_add(x, 0.3, s, residual=b, out=b), want)
    assert torch.equal(moe.moe_dropout_add(x, 0.3, s, residual=x), moe.moe_dropout_add(x, 0.3, s, residual=x.clone()))
    # the map is linear in x with a diagonal of 0 and 1 / (1 - p): the gradient is the map itself
    one = moe.moe_dropout_add(torch.ones((33, 130), device=DEV), 0.3, s)
    dy = torch.randn((33, 130), device=DEV)
    dx = moe.moe_dropout_add(dy, 0.3, s)
    assert torch.equal(dx, torch.where(one > 0, dy * one, torch.zeros_like(dy)))


def test_parts_of_a_tensor_and_offsets():
    """A call on the second half with its counters' offset gives the whole call's second half."""
    banner("dropout offsets")
    x = torch.randn(2 * 4096, device=DEV)
    whole = moe.moe_dropout_add(x, 0.4, rng(5, 100))
    half = moe.moe_dropout_add(x[4096:], 0.4, rng(5, 100 + moe.dropout_counters(4096)))
    assert torch.equal(whole[4096:], half)


def test_graph_reads_the_state_of_the_replay():
    banner("dropout graph")
    x, s = torch.randn(5000, device=DEV), rng(1, 0)
    y = torch.empty_like(x)
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        moe.moe_dropout_add(x, 0.2, s, out=y)
    torch.cuda.current_stream().wait_stream(st)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.moe_dropout_add(x, 0.2, s, out=y)
        s[1] += moe.dropout_counters(5000)
    for i in range(3):
        want = moe.moe_dropout_add(x, 0.2, rng(1, 1250 * i))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)


def test_large():
    """More elements than the grid has threads, an odd number."""
    banner("dropout large")
    n = 40_000_003
    x = torch.ones(n, device=DEV, dtype=BF)
    y = moe.moe_dropout_add(x, 0.25, rng(77, 3))
    at = 39_999_996
    words = O.dropout_words(8, 77, 3 + at // 4)[: n - at]
    assert np.array_equal((y[at:] != 0).cpu().numpy(), words >= np.uint64(1 << 30))
    kept = float((y != 0).double().mean())
    assert abs(kept - 0.75) < 5 * (0.1875 / n) ** 0.5
