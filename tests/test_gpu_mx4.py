"""GPU tests of MXFP4: quantisation, values, grouped products and the expert FFN.

Rules (fixed before any GPU run):
* quantisation and values: bit for bit the oracle's.
* products: a product of two E2M1 values and their power-of-two scales is exact
  in fp32, so an output differs from the exact sum by its fp32 additions in some
  order, at most K 2^-24 sum |a_i b_i|, and by one bf16 rounding (2^-9 of the
  value; 2^-8 allows for both sides of a rounding boundary).
* h: G and U differ from the exact ones by at most that bound; SiLU has slope at
  most 1.1, and its fp32 evaluation adds at most 2^-16 of h (the argument of the
  exponential carries |g| 2^-24, |g| < 100 here). With the scale code that the GPU
  wrote, each code's value lies between the roundings of h - bound and h + bound
  (rounding is monotone), and the scale code is one of those the bound allows.
* y: the product rule on the h that the GPU wrote.
* NaN and infinite tokens make their own rows NaN and no others.
"""
import numpy as np
import pytest
import torch

import paper_2606_00735_amd as moe
from oracle import mx4_oracle as Q

pytestmark = pytest.mark.gpu
DEV = "cuda"
REL = 2.0 ** -24


def banner(*a):
    print("CASE", *a, flush=True)


def mx4(codes, scales):
    """Mx4Tensor of oracle codes and scale codes."""
    b, d = Q.pack(codes, scales)
    return moe.Mx4Tensor(torch.from_numpy(b).to(DEV), torch.from_numpy(d).to(DEV), codes.shape[-1])


def unpacked(t):
    return Q.unpack(t.codes.cpu().numpy(), t.scales.cpu().numpy(), t.K)


def values64(t):
    q, s = unpacked(t)
    return torch.from_numpy(Q.values(q, s)).to(DEV)


def random_mx4(r, shape, spread=3):
    q = r.integers(0, 16, shape).astype(np.uint8)
    s = (r.integers(-spread, spread + 1, shape[:-1] + (shape[-1] // 32,)) + 120).astype(np.uint8)
    return mx4(q, s)


def offsets_of(rows):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)).to(DEV)


# ---------------------------------------------------------------- quantisation
def special(r, R, K):
    """Rows of blocks that test each rule: sizes over the whole exponent range,
    ties, zeros of both signs, denormals, the largest values, NaN, infinities."""
    x = r.standard_normal((R, K // 32, 32)) * np.exp2(r.integers(-140, 120, (R, K // 32, 1)).astype(float))
    flat = x.reshape(-1, 32)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.9, 0.0, -0.0, -0.25, -2.5, -5.0, -7.0, 0.1])
    for i in range(flat.shape[0]):
        if i % 7 == 1:
            flat[i] = np.concatenate([[4.0], r.choice(ties, 31)]) * 2.0 ** r.integers(-126, 120)
        elif i % 7 == 2:
            flat[i] = 0.0 if i % 2 else -0.0
        elif i % 7 == 3:
            flat[i] = r.choice([1e-45, -1e-44, 3e-40, 1e-39, 2.0 ** -126, -2.0 ** -127], 32)
        elif i % 7 == 4:
            flat[i] = r.choice([3.4e38, -3.3e38, 1e38, 1.0], 32)
        elif i % 7 == 5:
            flat[i, r.integers(32)] = r.choice([np.nan, np.inf, -np.inf])
    return torch.from_numpy(flat.reshape(R, K)).float()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("R,K", [(1, 32), (5, 96), (16, 256), (17, 288), (33, 512), (15, 544), (333, 4224), (64, 7168)])
def test_quantize_and_values(dtype, R, K):
    banner("quantize", dtype, R, K)
    x = special(np.random.default_rng(R + K), R, K).to(dtype)
    t = moe.moe_mx4_quantize(x.to(DEV))
    v = moe.moe_mx4_dequantize(t)
    q, s = Q.quantize(x.float().numpy())
    b, d = Q.pack(q, s)
    assert np.array_equal(t.scales.cpu().numpy(), d)
    assert np.array_equal(t.codes.cpu().numpy(), b)
    want, got = Q.values(q, s), v.float().cpu().numpy().astype(np.float64)
    assert np.array_equal(np.isnan(want), np.isnan(got))
    ok = ~np.isnan(want)
    assert np.array_equal(want[ok], got[ok]) and np.array_equal(np.signbit(want[ok]), np.signbit(got[ok]))


def test_values_of_every_code_and_scale():
    banner("values of all codes")
    s = np.repeat(np.arange(0, 256, dtype=np.uint8), 1).reshape(256, 1)
    q = np.tile(np.arange(16, dtype=np.uint8), 2)[None].repeat(256, 0)
    v = moe.moe_mx4_dequantize(mx4(q, s)).float().cpu().numpy().astype(np.float64)
    want = Q.values(q, s)
    assert np.isnan(v[255]).all()
    assert np.array_equal(v[:253], want[:253])


def test_quantize_batch_padded_rows_and_row_count():
    banner("quantize batch, ld, row_count")
    r = np.random.default_rng(3)
    x = torch.from_numpy(r.standard_normal((3, 20, 320))).float()
    q, s = Q.quantize(x.numpy())
    b, d = Q.pack(q, s)
    t = moe.moe_mx4_quantize(x.to(DEV), ld=272)
    assert t.ld == 272 and np.array_equal(t.codes.cpu().numpy(), b) and np.array_equal(t.scales.cpu().numpy(), d)
    assert np.array_equal(moe.moe_mx4_dequantize(t).float().cpu().numpy(), Q.values(q, s))
    for n in (0, 1, 13, 20, 99, -4):
        t = moe.Mx4Tensor(torch.full((20, 256), 0x5A, dtype=torch.uint8, device=DEV),
                          torch.full((2, 20, 2), 0x11111111, dtype=torch.int32, device=DEV), 320)
        moe.moe_mx4_quantize(x[0].to(DEV), out=t, row_count=torch.tensor([n], dtype=torch.int32, device=DEV))
        m = min(max(n, 0), 20)
        assert np.array_equal(t.codes.cpu().numpy()[:m], b[0, :m]) and (t.codes[m:] == 0x5A).all()
        assert np.array_equal(t.scales.cpu().numpy()[:, :m], d[0][:, :m]) and (t.scales[:, m:] == 0x11111111).all()


def test_quantize_empty():
    t = moe.moe_mx4_quantize(torch.empty((0, 256), device=DEV))
    assert t.shape == (0, 256) and moe.moe_mx4_dequantize(t).shape == (0, 256)


# ---------------------------------------------------------------- products
GEMM_CASES = [
    # N, K, rows per expert: every tile class with ragged tails, empty experts
    (128, 128, [1]),
    (384, 384, [63, 0, 64, 65]),
    (256, 2048, [128, 129, 0, 255, 256, 257]),
    (768, 4224, [300, 0, 1, 7]),
    (1024, 512, [8192]),
    (4096, 768, [4097, 3]),
]


@pytest.mark.parametrize("N,K,rows", GEMM_CASES)
def test_grouped_gemm(N, K, rows):
    banner("gemm", N, K, rows)
    r = np.random.default_rng(N + K)
    m = sum(rows)
    a, b = random_mx4(r, (m + 5, K)), random_mx4(r, (len(rows), N, K))
    c = torch.full((m + 5, N), float("nan"), dtype=torch.bfloat16, device=DEV)
    moe.moe_grouped_gemm_mx4(a, b, offsets_of(rows), c=c)
    va, vb = values64(a), values64(b)
    r0 = 0
    for e, n in enumerate(rows):
        if n:
            x = va[r0:r0 + n]
            want, mag = x @ vb[e].T, x.abs() @ vb[e].abs().T
            d = (c[r0:r0 + n].double() - want).abs()
            assert (d <= K * REL * mag + 2.0 ** -8 * want.abs()).all(), (e, float((d / mag).max()))
        r0 += n
    assert torch.isnan(c[m:]).all(), "rows past the last expert are left alone"


def test_gemm_offsets_past_the_rows_are_clamped():
    banner("gemm clamp")
    r = np.random.default_rng(5)
    a, b = random_mx4(r, (40, 256)), random_mx4(r, (2, 128, 256))
    good = moe.moe_grouped_gemm_mx4(a, b, torch.tensor([0, 30, 40], dtype=torch.int32, device=DEV))
    got = moe.moe_grouped_gemm_mx4(a, b, torch.tensor([-3, 30, 1 << 30], dtype=torch.int32, device=DEV))
    assert torch.equal(good, got)


def test_padding_codes_of_activations_do_not_matter():
    """K = 128 mod 256: the second half of the last chunk of a row is padding."""
    banner("gemm padding")
    r = np.random.default_rng(6)
    a, b = random_mx4(r, (70, 384)), random_mx4(r, (1, 128, 384))
    off = offsets_of([70])
    want = moe.moe_grouped_gemm_mx4(a, b, off)
    a.codes[:, 192:] = 0xA7
    a.scales[1] |= torch.tensor(0x64640000, dtype=torch.int32, device=DEV)
    assert torch.equal(moe.moe_grouped_gemm_mx4(a, b, off), want)


def test_gemm_padded_weight_rows():
    banner("gemm ld")
    r = np.random.default_rng(7)
    a, b = random_mx4(r, (33, 512)), random_mx4(r, (3, 256, 512))
    off = offsets_of([10, 0, 23])
    wide = torch.full((3, 256, 256 + 128), 0xFF, dtype=torch.uint8, device=DEV)
    wide[:, :, :256] = b.codes
    got = moe.moe_grouped_gemm_mx4(a, moe.Mx4Tensor(wide[:, :, :256], b.scales, 512), off)
    assert torch.equal(got, moe.moe_grouped_gemm_mx4(a, b, off))


# ---------------------------------------------------------------- FFN
def round_at(v, c):
    """Values of v rounded to E2M1 under scale codes c [.., K / 32] (float64, GPU)."""
    s = torch.exp2(c.double() - 127.0).repeat_interleave(32, -1)
    t = (v / s).clamp(-6.0, 6.0)
    step = torch.where(t.abs() >= 4, 2.0, torch.where(t.abs() >= 2, 1.0, 0.5)).to(t.dtype)
    return torch.round(t / step) * step * s


def scale_codes(top):
    e = torch.frexp(top)[1] - 1
    return torch.where(top > 0, (e + 125).clamp(min=0), torch.zeros_like(e))


def check_h(h, x, wg, wu, rows):
    vh = values64(h)
    _, s = unpacked(h)
    s = torch.from_numpy(s.astype(np.int64)).to(DEV)
    H, r0 = x.shape[1], 0
    for e, n in enumerate(rows):
        if n:
            v = x[r0:r0 + n]
            G, U = v @ wg[e].T, v @ wu[e].T
            bG, bU = H * REL * (v.abs() @ wg[e].abs().T), H * REL * (v.abs() @ wu[e].abs().T)
            act = G / (1 + torch.exp(-G))
            want = act * U
            tol = 1.1 * bG * U.abs() + act.abs() * bU + 1.1 * bG * bU + 2.0 ** -16 * want.abs()
            lo, hi = want - tol, want + tol
            big = torch.maximum(lo.abs(), hi.abs()).unflatten(-1, (-1, 32)).amax(-1)
            low = torch.where(lo * hi > 0, torch.minimum(lo.abs(), hi.abs()), torch.zeros_like(lo))
            low = low.unflatten(-1, (-1, 32)).amax(-1)
            c = s[r0:r0 + n]
            assert ((c >= scale_codes(low)) & (c <= scale_codes(big))).all(), e
            got = vh[r0:r0 + n]
            assert ((got >= round_at(lo, c)) & (got <= round_at(hi, c))).all(), e
        r0 += n
    return vh


def ffn_h(ws, M_cap, I):
    """The h that an FFN call left in its workspace."""
    row, C = 128 * moe.mx4_chunks(I), moe.mx4_chunks(I)
    a = moe.FFN_COUNTER_BYTES
    b = a + (M_cap * row + 255) // 256 * 256
    return moe.Mx4Tensor(ws[a:a + M_cap * row].view(M_cap, row),
                         ws[b:b + C * M_cap * 8].view(torch.int32).view(C, M_cap, 2), I)


def make_ffn(r, H, I, n):
    def w(rows, K):
        v = (r.standard_normal((n, rows, K)) / np.sqrt(K)).astype(np.float32)
        return moe.moe_mx4_quantize(torch.from_numpy(v).to(DEV))
    return w(I, H), w(I, H), w(H, I)


def check_ffn(x, perm_src, k, w, rows, y, ws, M_cap, I):
    """x: Mx4Tensor of tokens (or rows); every stage of one FFN call."""
    m = sum(rows)
    vx = values64(x)
    vx = vx[:m] if perm_src is None else vx[(perm_src[:m] // k).long()]
    vg, vu, vd = (values64(t) for t in w)
    h = check_h(ffn_h(ws, M_cap, I), vx, vg, vu, rows)
    assert (ws[:moe.FFN_COUNTER_BYTES] == 0).all(), "counters are left zero"
    r0 = 0
    for e, n in enumerate(rows):
        if n:
            v = h[r0:r0 + n]
            want, mag = v @ vd[e].T, v.abs() @ vd[e].abs().T
            d = (y[r0:r0 + n].double() - want).abs()
            assert (d <= I * REL * mag + 2.0 ** -8 * want.abs()).all(), (e, float((d / mag).max()))
        r0 += n


FFN_CASES = [
    # H, I, rows per expert: decode (one row to 128), rounds, split launches, large tiles
    (256, 128, [1]),
    (2048, 768, [1] * 8 + [0] * 8),
    (2048, 768, [3, 0, 16, 17, 1, 64, 5, 2]),
    (4096, 1024, [128]),
    (4096, 384, [100, 28]),
    (2048, 768, [129, 0, 300, 65, 1]),
    (4096, 2048, [260, 70]),
    (7168, 2048, [520, 0, 1030]),
    (4096, 896, [2500]),
]


@pytest.mark.parametrize("H,I,rows", FFN_CASES)
def test_ffn(H, I, rows):
    banner("ffn", H, I, rows)
    r = np.random.default_rng(H + I + sum(rows))
    m = sum(rows)
    M_cap = m if m <= 128 else m + 3
    x = moe.moe_mx4_quantize(torch.from_numpy(r.standard_normal((M_cap, H))).float().to(DEV))
    w, off = make_ffn(r, H, I, len(rows)), offsets_of(rows)
    y = torch.full((M_cap, H), float("nan"), dtype=torch.bfloat16, device=DEV)
    _, ws = moe.moe_grouped_swiglu_ffn_mx4(x, *w, off, y_perm=y)
    check_ffn(x, None, 1, w, rows, y, ws, M_cap, I)
    assert torch.isnan(y[m:]).all()
    first = y.clone()
    for _ in range(3):
        moe.moe_grouped_swiglu_ffn_mx4(x, *w, off, y_perm=y, ws=ws)
        assert torch.equal(y[:m], first[:m]), "a repeated call differs"
    # the two halves by themselves
    h = moe.moe_grouped_swiglu_mx4(x, w[0], w[1], off)
    vh = check_h(h, values64(x)[:m], values64(w[0]), values64(w[1]), rows)
    assert vh.shape[0] == M_cap


FEW_CASES = [
    # H, I, rows per expert: calls of at most 128 rows and little weight. K of one chunk
    # and not a multiple of one, h rows that end inside a chunk, tiles of 16 rows with
    # ragged ends, experts past a wavefront's 64, more tiles than a grid holds, and the
    # first call with a row too many
    (128, 128, [1]),
    (384, 640, [0, 0, 2, 0]),
    (2048, 768, [1, 15, 16, 17, 33]),
    (7168, 256, [128]),
    (1152, 384, [0] * 63 + [5, 1] + [0] * 62 + [2, 0, 3]),
    (256, 1024, [1, 0] * 127 + [1, 0]),
    (256, 2048, [0, 1] * 100 + [28]),
    (2048, 384, [100, 29]),
]


@pytest.mark.parametrize("H,I,rows", FEW_CASES)
def test_ffn_few_rows(H, I, rows):
    banner("ffn few", H, I, len(rows), sum(rows))
    r = np.random.default_rng(H + I + len(rows))
    m = sum(rows)
    x = moe.moe_mx4_quantize(torch.from_numpy(r.standard_normal((m, H))).float().to(DEV))
    w, off = make_ffn(r, H, I, len(rows)), offsets_of(rows)
    y, ws = moe.moe_grouped_swiglu_ffn_mx4(x, *w, off)
    check_ffn(x, None, 1, w, rows, y, ws, m, I)
    # each half by itself does the same work
    h = moe.moe_grouped_swiglu_mx4(x, w[0], w[1], off)
    q1, q2 = unpacked(h), unpacked(ffn_h(ws, m, I))
    assert np.array_equal(q1[0], q2[0]) and np.array_equal(q1[1], q2[1])
    assert torch.equal(moe.moe_grouped_gemm_mx4(h, w[2], off), y)


@pytest.mark.parametrize("m", [5, 20, 100])
def test_ffn_few_rows_empty_and_foreign_offsets(m):
    """No rows at all; and offsets that run backwards or out of the buffer, which every
    expert reads clamped to it: the last writer of a row wins, all values stay finite."""
    banner("ffn few offsets", m)
    r = np.random.default_rng(m)
    x = moe.moe_mx4_quantize(torch.from_numpy(r.standard_normal((m, 512))).float().to(DEV))
    w = make_ffn(r, 512, 384, 3)
    y = torch.full((m, 512), float("nan"), dtype=torch.bfloat16, device=DEV)
    moe.moe_grouped_swiglu_ffn_mx4(x, *w, offsets_of([0, 0, 0]), y_perm=y)
    assert torch.isnan(y).all()
    off = torch.tensor([-7, m, 1, 1 << 30], dtype=torch.int32, device=DEV)
    moe.moe_grouped_swiglu_ffn_mx4(x, *w, off, y_perm=y)
    assert torch.isfinite(y.float()).all()


def route(r, T, k, E, E_local):
    ids = np.stack([r.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    emap = np.full(E, -1, np.int32)
    emap[r.permutation(E)[:E_local]] = np.arange(E_local)
    t = torch.from_numpy(ids).to(DEV)
    counts, offsets, ws = moe.moe_expert_histogram_scan(t, E, emap)
    _, perm_src, dest = moe.moe_permute(torch.empty((T, 8), dtype=torch.bfloat16, device=DEV), t, emap, ws, gather=False)
    return perm_src, offsets, np.diff(offsets.cpu().numpy()).tolist()


@pytest.mark.parametrize("T,k,E,E_local,H,I", [(1, 2, 8, 8, 2048, 768), (9, 4, 16, 4, 512, 384), (127, 8, 32, 32, 2048, 768),
                                               (700, 8, 16, 16, 2048, 768), (3000, 2, 16, 4, 4096, 512)])
def test_ffn_gather(T, k, E, E_local, H, I):
    """Rows read through perm_src, by the rules and against the permuted rows."""
    banner("ffn gather", T, k, E, E_local, H, I)
    r = np.random.default_rng(T)
    perm_src, off, rows = route(r, T, k, E, E_local)
    m = sum(rows)
    x = moe.moe_mx4_quantize(torch.from_numpy(r.standard_normal((T, H))).bfloat16().to(DEV))
    w = make_ffn(r, H, I, E_local)
    y, ws = moe.moe_grouped_swiglu_ffn_mx4(x, *w, off, perm_src=perm_src, k=k)
    check_ffn(x, perm_src, k, w, rows, y, ws, T * k, I)
    y2, _ = moe.moe_grouped_swiglu_ffn_mx4(x, *w, off, perm_src=perm_src, k=k, experts=E, ws=ws)
    tok = (perm_src[:m] // k).long()
    xp = moe.Mx4Tensor(x.codes[tok].contiguous(), x.scales[:, tok].contiguous(), H)
    h1 = moe.moe_grouped_swiglu_mx4(x, w[0], w[1], off, perm_src=perm_src, k=k)
    h2 = moe.moe_grouped_swiglu_mx4(xp, w[0], w[1], off)
    q1, q2 = unpacked(h1), unpacked(h2)
    assert np.array_equal(q1[0][:m], q2[0][:m]) and np.array_equal(q1[1][:m], q2[1][:m])
    d = (y2[:m].double() - y[:m].double()).norm() / y[:m].double().norm()
    assert d <= 1e-2


def test_ffn_nan_and_infinite_tokens():
    banner("ffn nan")
    r = np.random.default_rng(11)
    H, I, rows = 512, 384, [40, 30]
    v = torch.from_numpy(r.standard_normal((70, H))).float()
    clean = moe.moe_mx4_quantize(v.to(DEV))
    v[3, 17], v[50, 400], v[69, 0] = float("nan"), float("inf"), float("-inf")
    x = moe.moe_mx4_quantize(v.to(DEV))
    w, off = make_ffn(r, H, I, 2), offsets_of(rows)
    y, _ = moe.moe_grouped_swiglu_ffn_mx4(x, *w, off)
    want, _ = moe.moe_grouped_swiglu_ffn_mx4(clean, *w, off)
    bad = torch.zeros(70, dtype=torch.bool, device=DEV)
    bad[[3, 50, 69]] = True
    assert torch.isnan(y[bad]).all() and torch.equal(y[~bad], want[~bad])


def test_ffn_no_rows():
    banner("ffn empty")
    r = np.random.default_rng(12)
    w = make_ffn(r, 256, 256, 3)
    x = moe.moe_mx4_quantize(torch.randn((20, 256), device=DEV))
    y = torch.full((20, 256), 7.0, dtype=torch.bfloat16, device=DEV)
    _, ws = moe.moe_grouped_swiglu_ffn_mx4(x, *w, offsets_of([0, 0, 0]), y_perm=y)
    assert (y == 7.0).all() and (ws[:moe.FFN_COUNTER_BYTES] == 0).all()


def test_ffn_other_stream_and_graph():
    """Launches on the current stream only, and under capture: replays on new
    contents of the same buffers equal eager calls."""
    banner("ffn stream, graph")
    r = np.random.default_rng(13)
    for rows in ([5, 9, 0, 2], [200, 0, 300, 1]):
        m, H, I = sum(rows), 2048, 768
        w, off = make_ffn(r, H, I, 4), offsets_of(rows)
        vs = [torch.from_numpy(r.standard_normal((m, H))).bfloat16().to(DEV) for _ in range(3)]
        eager = [moe.moe_grouped_swiglu_ffn_mx4(moe.moe_mx4_quantize(v), *w, off)[0] for v in vs]
        src, y = vs[0].clone(), torch.empty((m, H), dtype=torch.bfloat16, device=DEV)
        q = moe.moe_mx4_quantize(src)
        ws = torch.zeros(moe.ffn_mx4_ws_bytes(4, H, I, m), dtype=torch.uint8, device=DEV)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            moe.moe_mx4_quantize(src, out=q)
            moe.moe_grouped_swiglu_ffn_mx4(q, *w, off, ws=ws, y_perm=y)
        s.synchronize()
        assert torch.equal(y, eager[0])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            moe.moe_mx4_quantize(src, out=q)
            moe.moe_grouped_swiglu_ffn_mx4(q, *w, off, ws=ws, y_perm=y)
        for i in (1, 2, 0, 1):
            src.copy_(vs[i])
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(y, eager[i]), i


# ---------------------------------------------------------------- refusals
def test_refusals():
    banner("refusals")
    x = torch.randn((4, 256), device=DEV)
    t = moe.moe_mx4_quantize(x)
    w = moe.moe_mx4_quantize(torch.randn((2, 128, 256), device=DEV))
    off = offsets_of([2, 2])
    with pytest.raises(ValueError):
        moe.moe_mx4_quantize(torch.randn((4, 48), device=DEV))
    with pytest.raises(ValueError):
        moe.moe_mx4_quantize(x.half())
    with pytest.raises(ValueError):
        moe.moe_mx4_quantize(torch.randn((256, 4), device=DEV).t())
    with pytest.raises(ValueError):
        moe.moe_mx4_quantize(x, out=moe.moe_mx4_quantize(torch.randn((5, 256), device=DEV)))
    with pytest.raises(ValueError):
        moe.Mx4Tensor(t.codes, t.scales, 512)
    with pytest.raises(ValueError):
        moe.moe_grouped_gemm_mx4(t, w, offsets_of([4]))
    with pytest.raises(ValueError):
        moe.moe_grouped_gemm_mx4(moe.moe_mx4_quantize(torch.randn((4, 512), device=DEV)), w, off)
    with pytest.raises(TypeError):
        moe.moe_grouped_swiglu_ffn_mx4(x, w, w, w, off)
    odd = moe.moe_mx4_quantize(torch.randn((1, 96, 256), device=DEV))
    with pytest.raises(moe.MoeError):
        moe.moe_grouped_gemm_mx4(t, odd, offsets_of([4]))
    wd = moe.moe_mx4_quantize(torch.randn((2, 256, 128), device=DEV))
    with pytest.raises(moe.MoeError) as e:
        moe.moe_grouped_swiglu_ffn_mx4(t, w, w, wd, off, ws=torch.zeros(1024, dtype=torch.uint8, device=DEV))
    assert e.value.status == 3
    with pytest.raises(moe.MoeError):
        moe.moe_grouped_swiglu_ffn_mx4(t, w, w, wd, off, perm_src=torch.zeros(4, dtype=torch.int32, device=DEV), k=0)
    with pytest.raises(ValueError):
        moe.moe_grouped_swiglu_ffn_mx4(t, w, w, wd, off, experts=1)
