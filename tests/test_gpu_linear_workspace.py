"""GPU test: one workspace, sized for the largest batch, serves every smaller one and gives the
bits of a workspace of the call's own; what it held before does not matter."""
import pytest
import torch

import paper_2606_00735_amd as moe

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF = torch.bfloat16


@pytest.mark.parametrize("N,K", [(1024, 4096), (4096, 1024), (264, 8200), (768, 2048)])
def test_one_workspace_for_all_batches(N, K):
    print("CASE linear workspace", N, K, flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(N)
    most = 4096
    fw = torch.empty(moe.linear_ws_bytes(most, N, K, BF) + 256, dtype=torch.uint8, device=DEV)
    bw = torch.empty(moe.linear_backward_ws_bytes(most, N, K, BF) + 256, dtype=torch.uint8, device=DEV)
    w = (torch.randn((N, K), generator=g, device=DEV) / K ** 0.5).to(BF)
    for M in (most, 2000, 1025, 1000, 513, 300, 100, 40, 9, 1):
        x, dy = (torch.randn((M, n), generator=g, device=DEV).to(BF) for n in (K, N))
        for t in (fw, bw):
            t.fill_(255)
        y = moe.moe_linear(x, w, residual=dy, ws=fw[:-256])
        assert torch.equal(y, moe.moe_linear(x, w, residual=dy)), M
        got = moe.moe_linear_backward(dy, x, w, z=y, act="silu", ws=bw[:-256])
        want = moe.moe_linear_backward(dy, x, w, z=y, act="silu")
        assert all(torch.equal(a, b) for a, b in zip(got[:4], want[:4])), M
        got, want = moe.moe_linear_backward(dy, x, w, ws=bw[:-256]), moe.moe_linear_backward(dy, x, w)
        assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3])), M
        assert (fw[-256:] == 255).all() and (bw[-256:] == 255).all()
