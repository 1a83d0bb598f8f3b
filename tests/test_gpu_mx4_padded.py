"""GPU test of MXFP4 quantisation into padded rows of batches of single rows, bit for bit the oracle's."""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import mx4_oracle as Q

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,R,K,ld", [(3, 1, 320, 272), (5, 1, 32, 144), (1, 1, 512, 272), (2, 2, 256, 128)])
def test_quantize_single_rows_with_a_stride(B, R, K, ld):
    print("CASE quantize single rows", B, R, K, ld, flush=True)
    x = torch.from_numpy(np.random.default_rng(K).standard_normal((B, R, K))).float()
    q, s = Q.quantize(x.numpy())
    b, d = Q.pack(q, s)
    t = moe.moe_mx4_quantize(x.cuda(), ld=ld)
    assert np.array_equal(t.codes.cpu().numpy(), b) and np.array_equal(t.scales.cpu().numpy(), d)
    assert np.array_equal(moe.moe_mx4_dequantize(t).float().cpu().numpy(), Q.values(q, s))
