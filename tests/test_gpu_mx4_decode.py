"""GPU tests of the MXFP4 FFN where experts have few rows and the weights are many, the
decode schedule, alone and beside the kernel of few rows, each against float64.

A call takes the kernel of few rows for a product of at most 128 rows and 128 MB of
codes, counted once per tile of 16 rows; gate/up has two matrices and down one, so the
two halves of a call may differ. All other products of experts of at most 16 rows take
the decode schedule.

Tolerances (fixed before any GPU run): those of test_gpu_mx4 (K 2^-24 of the products'
sizes for a sum, one bf16 rounding; h's codes between the roundings of h - bound and h +
bound under the scale that the GPU wrote).
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import mx4_oracle as Q

pytestmark = pytest.mark.gpu
DEV = "cuda"
REL = 2.0 ** -24
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def banner(*a):
    print("CASE", *a, flush=True)


def values(codes, scales, K):
    """(float64 values [R, K], scale codes [R, K / 32]) of one matrix, on the GPU."""
    q = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).long()
    v = torch.tensor(GRID + tuple(-x for x in GRID), dtype=torch.float64, device=DEV)[q]
    s = (scales.unsqueeze(-1) >> torch.arange(0, 32, 8, device=DEV)) & 255  # [C, R, h, s]: block 2 s + h
    s = s.permute(1, 0, 3, 2).reshape(codes.shape[0], -1)
    v = v.unflatten(-1, (-1, 32)) * torch.exp2(s.double() - 127.0).unsqueeze(-1)
    return v.flatten(-2)[:, :K], s[:, : K // 32].long()


def test_values_are_the_oracles():
    banner("values")
    r = np.random.default_rng(1)
    for R, K in ((3, 32), (5, 384), (2, 544)):
        q, s = r.integers(0, 16, (R, K)).astype(np.uint8), r.integers(0, 255, (R, K // 32)).astype(np.uint8)
        b, d = Q.pack(q, s)
        v, c = values(torch.from_numpy(b).to(DEV), torch.from_numpy(d).to(DEV), K)
        assert np.array_equal(v.cpu().numpy(), Q.values(q, s)) and np.array_equal(c.cpu().numpy(), s)


def random_weights(n, rows, K, g):
    w = moe.Mx4Tensor(torch.empty((n, rows, 128 * moe.mx4_chunks(K)), dtype=torch.uint8, device=DEV),
                      torch.empty((n, moe.mx4_chunks(K), rows, 2), dtype=torch.int32, device=DEV), K)
    for e in range(n):
        m = torch.randn((rows, K), generator=g, device=DEV) / K ** 0.5
        moe.moe_mx4_quantize(m, out=moe.Mx4Tensor(w.codes[e], w.scales[e], K))
    return w


def round_at(v, c):
    s = torch.exp2(c.double() - 127.0).repeat_interleave(32, -1)
    t = (v / s).clamp(-6.0, 6.0)
    step = torch.where(t.abs() >= 4, 2.0, torch.where(t.abs() >= 2, 1.0, 0.5)).to(t.dtype)
    return torch.round(t / step) * step * s


def scale_codes(top):
    e = torch.frexp(top)[1] - 1
    return torch.where(top > 0, (e + 125).clamp(min=0), torch.zeros_like(e))


def check(x, tokens, w, offsets, y, ws, M_cap):
    """Every stage of one call: h as the workspace holds it, and y. tokens: the row of x
    behind each row."""
    H, I = x.shape[1], w[0].shape[1]
    C = moe.mx4_chunks(I)
    a = moe.FFN_COUNTER_BYTES
    assert not ws[:a].any(), "counters are left zero"
    b = a + (M_cap * 128 * C + 255) // 256 * 256
    vh, sh = values(ws[a:a + M_cap * 128 * C].view(M_cap, 128 * C),
                    ws[b:b + C * M_cap * 8].view(torch.int32).view(C, M_cap, 2), I)
    vx = values(x.codes, x.scales, H)[0][tokens]
    b = offsets.tolist()
    for e in range(len(b) - 1):
        if b[e] == b[e + 1]:
            continue
        at = slice(b[e], b[e + 1])
        wg, wu, wd = (values(t.codes[e], t.scales[e], t.K)[0] for t in w)
        G, U = vx[at] @ wg.T, vx[at] @ wu.T
        bG, bU = H * REL * (vx[at].abs() @ wg.abs().T), H * REL * (vx[at].abs() @ wu.abs().T)
        act = G / (1 + torch.exp(-G))
        want = act * U
        tol = 1.1 * bG * U.abs() + act.abs() * bU + 1.1 * bG * bU + 2.0 ** -16 * want.abs()
        lo, hi = want - tol, want + tol
        big = torch.maximum(lo.abs(), hi.abs()).unflatten(-1, (-1, 32)).amax(-1)
        low = torch.where(lo * hi > 0, torch.minimum(lo.abs(), hi.abs()), torch.zeros_like(lo)).unflatten(-1, (-1, 32)).amax(-1)
        c = sh[at]
        assert ((c >= scale_codes(low)) & (c <= scale_codes(big))).all(), e
        assert ((vh[at] >= round_at(lo, c)) & (vh[at] <= round_at(hi, c))).all(), e
        want, mag = vh[at] @ wd.T, vh[at].abs() @ wd.abs().T
        assert ((y[at].double() - want).abs() <= I * REL * mag + 2.0 ** -8 * want.abs()).all(), e


def run(x, w, offsets, M_cap, perm_src=None, k=1, **kw):
    m = int(offsets[-1])
    y = torch.full((M_cap, x.shape[1]), float("nan"), dtype=torch.bfloat16, device=DEV)
    _, ws = moe.moe_grouped_swiglu_ffn_mx4(x, *w, offsets, y_perm=y, perm_src=perm_src, k=k, **kw)
    tokens = torch.arange(m, device=DEV) if perm_src is None else (perm_src[:m] // k).long()
    check(x, tokens, w, offsets, y, ws, M_cap)
    assert torch.isnan(y[m:]).all()
    return y[:m], ws


CASES = [
    # H, I, rows per expert, rows of room
    (512, 384, [1, 0, 16, 7, 3] * 4, 200),                  # up to 16 rows, small weights, too many rows for few
    (2048, 768, [9, 16, 1, 12, 0, 2, 15, 8] * 2, 129),      # the same by one row of room
    (640, 1152, [16] * 13, 208),                            # rows of K and h that end inside a chunk
    (4096, 14336, [8] * 8, 64),                             # a decode batch: both halves
    (4096, 8320, [1, 5, 0, 16, 2, 9, 3, 11], 47),           # ragged; a bit more than 128 MB in down
    (7168, 5120, [64], 64),                                 # one expert: gate/up by the decode schedule, down few
    (2048, 768, [1] * 128, 128),                            # gate/up by the decode schedule, down few
    (2048, 768, [3, 0, 1, 2] * 16 + [0] * 64, 120),
    (2048, 1280, [1] * 100 + [0] * 10 + [2] * 14, 128),     # both by the decode schedule
]


@pytest.mark.parametrize("H,I,rows,M_cap", CASES)
def test_ffn(H, I, rows, M_cap):
    banner("ffn", H, I, len(rows), sum(rows), M_cap)
    g = torch.Generator(device=DEV)
    g.manual_seed(H + I + M_cap)
    E = len(rows)
    x = moe.moe_mx4_quantize(torch.randn((M_cap, H), generator=g, device=DEV))
    w = [random_weights(E, I, H, g), random_weights(E, I, H, g), random_weights(E, H, I, g)]
    offsets = torch.tensor(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32), device=DEV)
    y, ws = run(x, w, offsets, M_cap)
    # a call of few rows and one of the decode schedule on one workspace, in turn
    few = [moe.Mx4Tensor(t.codes[:1], t.scales[:1], t.K) for t in w]
    one = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    x1 = moe.Mx4Tensor(x.codes[:1], x.scales[:, :1].contiguous(), H)
    want, _ = run(x1, few, one, 1)
    for _ in range(3):
        got, _ = moe.moe_grouped_swiglu_ffn_mx4(x1, *few, one, ws=ws)
        assert torch.equal(got, want)
        again, _ = moe.moe_grouped_swiglu_ffn_mx4(x, *w, offsets, ws=ws)
        assert torch.equal(again[: y.shape[0]], y), "a repeated call differs"
        assert not ws[: moe.FFN_COUNTER_BYTES].any()


@pytest.mark.parametrize("T,k,E,E_local,H,I", [
    (16, 8, 128, 128, 2048, 768),   # gate/up by the decode schedule, down few
    (2, 8, 256, 32, 7168, 2048),    # the same on a shard: most assignments are remote
    (4, 8, 256, 32, 7168, 2048),    # both by the decode schedule
    (4, 1, 128, 16, 5120, 8192),    # one expert a token
    (40, 4, 32, 16, 512, 384),      # more than 128 rows of room
    (13, 8, 32, 32, 2048, 768),     # few rows in both
])
def test_ffn_gather(T, k, E, E_local, H, I):
    """Routed rows of a shard, and the same rows permuted before; `experts` changes no bit."""
    banner("ffn gather", T, k, E, E_local, H, I)
    r = np.random.default_rng(T)
    ids = np.stack([r.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    if 0 not in ids[0]:
        ids[0, 0] = 0  # at least one assignment is local
    emap = np.full(E, -1, np.int32)
    emap[np.arange(E_local) * (E // E_local)] = r.permutation(E_local)
    t = torch.from_numpy(ids).to(DEV)
    _, offsets, hws = moe.moe_expert_histogram_scan(t, E, emap)
    _, perm_src, _ = moe.moe_permute(torch.empty((T, 8), dtype=torch.bfloat16, device=DEV), t, emap, hws, gather=False)
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    x = moe.moe_mx4_quantize(torch.randn((T, H), generator=g, device=DEV).bfloat16())
    w = [random_weights(E_local, I, H, g), random_weights(E_local, I, H, g), random_weights(E_local, H, I, g)]
    y, ws = run(x, w, offsets, T * k, perm_src=perm_src, k=k)
    m = y.shape[0]
    again, _ = moe.moe_grouped_swiglu_ffn_mx4(x, *w, offsets, perm_src=perm_src, k=k, experts=E, ws=ws)
    assert torch.equal(again[:m], y)
    tok = torch.zeros(T * k, dtype=torch.int64, device=DEV)
    tok[:m] = perm_src[:m] // k
    run(moe.Mx4Tensor(x.codes[tok].contiguous(), x.scales[:, tok].contiguous(), H), w, offsets, T * k)


def test_decode_schedule_in_a_graph():
    """Replays on new contents, of a call whose halves take different kernels."""
    banner("decode graph")
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    E, H, I = 128, 2048, 768
    w = [random_weights(E, I, H, g), random_weights(E, I, H, g), random_weights(E, H, I, g)]
    offsets = torch.arange(E + 1, dtype=torch.int32, device=DEV)
    vs = [torch.randn((E, H), generator=g, device=DEV).bfloat16() for _ in range(3)]
    want = [run(moe.moe_mx4_quantize(v), w, offsets, E)[0].clone() for v in vs]
    src, y = vs[0].clone(), torch.empty((E, H), dtype=torch.bfloat16, device=DEV)
    q = moe.moe_mx4_quantize(src)
    ws = torch.zeros(moe.ffn_mx4_ws_bytes(E, H, I, E), dtype=torch.uint8, device=DEV)
    moe.moe_grouped_swiglu_ffn_mx4(q, *w, offsets, ws=ws, y_perm=y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.moe_mx4_quantize(src, out=q)
        moe.moe_grouped_swiglu_ffn_mx4(q, *w, offsets, ws=ws, y_perm=y)
    for i in (1, 2, 0, 1):
        src.copy_(vs[i])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[i]), i
