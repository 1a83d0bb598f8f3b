"""GPU tests of the training calls at their largest token counts, where an index past 31
bits would show in the counts and at the ends of the outputs.

Tolerances (fixed before any GPU run), u = 2^-24: sums of terms of one sign in fp32
within a block, at most 64 additions a lane and 16 between lanes, the blocks in fp64:
relative 128 u, with exp and log to 2 ulp.
"""
import pytest
import torch

import paper_2606_00735_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24


def banner(*a):
    print("CASE", *a, flush=True)


@pytest.fixture(autouse=True)
def give_back():
    torch.cuda.empty_cache()
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T,seq", [(2 ** 31 - 256, 0), (2 ** 23 - 1, 1)])
def test_balance_at_the_block_limit(T, seq):
    """Two experts, every token with logits (0, log 3); the first of them from token 5 on."""
    banner("balance limit", T, seq)
    E, G = 2, T // seq if seq else 1
    z = torch.zeros((T, E), device=DEV)
    z[:, 1] = 1.0986122886681098
    ids = torch.zeros((T, 1), dtype=torch.int32, device=DEV)
    ids[:5] = 1
    loss, counts, live, ws = moe.moe_balance_loss(z, ids, seq_len=seq)
    lse = 2 * 0.6931471805599453
    want = [2 * (0.25 * (T - 5) + 0.75 * 5) / T, lse * lse]
    assert all(abs(float(a) - b) <= 128 * U * b for a, b in zip(loss, want)), (loss, want)
    assert live[:G].sum() == T and live[-2:].tolist() == [T, G] and not ws[:256].any()
    if seq:
        assert (counts[:5] == torch.tensor([0, 1], device=DEV)).all() and (counts[5:] == torch.tensor([1, 0], device=DEV)).all()
    else:
        assert counts.tolist() == [[T - 5, 5]]
    del ws
    d = moe.moe_gate_backward(z, ids, counts, live, torch.tensor([0.0, float(T)], device=DEV), seq_len=seq)
    want = 2 * lse * torch.tensor([0.25, 0.75], device=DEV)
    for at in (slice(0, 300), slice(T // 2, T // 2 + 300), slice(T - 300, T)):
        assert ((d[at] - want).abs() <= 128 * U * want).all()
