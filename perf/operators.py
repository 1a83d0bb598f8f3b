"""Timed cases of the 4-bit experts and of the router's training step: what a
program does that serves mixture-of-experts layers with MXFP4 experts, or
fine-tunes a router over them.

Kinds of case:

* ``quant``: MXFP4 quantisation of token rows or of a weight matrix, and the
  values that the codes stand for;
* ``ffn``: the MXFP4 expert FFN of one GPU's shard: token rows quantised, then
  the grouped SwiGLU FFN reading the routed rows;
* ``balance``: the balance and z losses of a router's logits, the per-expert
  counts, and the gradient to the logits (with the gate weights' own gradient);
* ``router``: the gradient of the router's product: to the router's weights,
  its bias and the tokens;
* ``combine``: the gradient of the weighted combine: to the gate weights and the
  experts' rows.

The layer shapes are the library's five workloads. ``own`` chooses between the
plain form (elementary torch operations in fp32) and the library's calls.
"""
import math

import torch

own = False

# name: H, I, E, k, experts on this GPU, largest T
SHAPES = {
    "tiny": (128, 256, 8, 2, 8, 64),
    "mixtral": (4096, 14336, 8, 2, 8, 4096),
    "qwen3": (2048, 768, 128, 8, 128, 8192),
    "dsv3_shard": (7168, 2048, 256, 8, 32, 16384),
    "maverick_shard": (5120, 8192, 128, 1, 16, 32768),
}
BIG = ("mixtral", "qwen3", "dsv3_shard", "maverick_shard")


def _ffn(name, shape, T, alpha):
    return {"name": name, "kind": "ffn", "shape": shape, "T": T, "alpha": alpha}


def listed():
    return [
        # a weight matrix of one expert held in fp32, quantised when it is loaded;
        # an odd number of rows of a length that is no whole number of chunks
        {"name": "quant_weight_fp32", "kind": "quant", "rows": 333, "K": 4224, "dtype": "fp32"},
        # the activations of the largest prefill batch
        {"name": "quant_tokens", "kind": "quant", "rows": 16384, "K": 7168, "dtype": "bf16"},
        # one token: eight experts with one row each, where launches and fills count
        _ffn("ffn_qwen3_token", "qwen3", 1, 1.0),
        # a decode batch: every expert's weights streamed
        _ffn("ffn_mixtral_decode", "mixtral", 32, 0.0),
        # a chunk of a prompt between decodes: about 60 ragged rows an expert
        _ffn("ffn_qwen3_chunk", "qwen3", 1000, 0.0),
        # a prefill batch of few large, skewed experts
        _ffn("ffn_mixtral_prefill", "mixtral", 4096, 1.0),
        # the smallest layer, one group
        {"name": "balance_tiny", "kind": "balance", "E": 8, "k": 2, "T": 64, "seq": 0, "pad": 0.0, "alpha": 1.0},
        # a training batch of padded sequences, the loss taken for each of them
        {"name": "balance_dsv3", "kind": "balance", "E": 256, "k": 8, "T": 16384, "seq": 4096, "pad": 0.2, "alpha": 1.0},
        # the fp32 layer at its only size
        {"name": "router_tiny_fp32", "kind": "router", "shape": "tiny", "T": 64},
        # the same training batch's router
        {"name": "router_dsv3", "kind": "router", "shape": "dsv3_shard", "T": 16384},
        # an odd micro-batch, every expert local
        {"name": "combine_qwen3_odd", "kind": "combine", "shape": "qwen3", "T": 777, "alpha": 1.0},
        # a shard's part of a large batch: one assignment of eight is local
        {"name": "combine_dsv3", "kind": "combine", "shape": "dsv3_shard", "T": 16384, "alpha": 0.0},
    ]


def _log_int(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n))


def draw(rng):
    kind = rng.choice(["quant", "ffn", "ffn", "balance", "router", "combine"])
    if kind == "quant":
        return {"kind": kind, "rows": _log_int(rng, 1, 16384), "K": 32 * _log_int(rng, 4, 448), "dtype": rng.choice(["bf16", "fp32"])}
    if kind == "balance":
        E, k = rng.choice([(8, 2), (60, 4), (128, 1), (128, 8), (256, 8)])
        seqs = rng.choice([0, 1, 2, 3, 4])
        T = _log_int(rng, 1, 16384)
        if seqs:  # whole sequences
            T = max(1, T // seqs) * seqs
        return {"kind": kind, "E": E, "k": k, "T": T, "seq": T // seqs if seqs else 0, "pad": rng.choice([0.0, 0.2, 0.9]), "alpha": rng.choice([0.0, 1.0, 1.5])}
    if kind == "router" and rng.random() < 0.2:
        return {"kind": kind, "shape": "tiny", "T": rng.randint(1, 64)}
    shape = rng.choice(BIG)
    T = _log_int(rng, 1, min(SHAPES[shape][5], 16384))
    if kind == "router":
        return {"kind": kind, "shape": shape, "T": T}
    if SHAPES[shape][2] > SHAPES[shape][4]:  # enough tokens that some of them are local
        T = max(T, 128)
    return {"kind": kind, "shape": shape, "T": T, "alpha": rng.choice([0.0, 1.0, 1.5])}


# ---------------------------------------------------------------------------
# MXFP4 in torch: 32 consecutive elements of a row share the power of two
# 2^(c - 127); two E2M1 codes a byte, the even element in the low half. A row is
# padded with zero codes to whole chunks of 256 elements; the 8 scale codes of a
# chunk are two words of 4 bytes, the even blocks' in the first, the odd
# blocks' in the second, [chunk][row][2].
# ---------------------------------------------------------------------------
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _padded(K):
    return (K + 255) // 256 * 256


def _blocks(v):
    """Scale codes [.., K/32] (as exponents + 127) and scaled elements [.., K/32, 32] of fp32 rows [.., K]."""
    b = v.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1)
    e = torch.frexp(top)[1] - 1  # floor(log2 top)
    c = torch.where(top > 0, (e - 2 + 127).clamp(0, 254), torch.zeros_like(e))
    # 2^(127 - c) may pass fp32's largest power of two: in two factors
    n = 127 - c
    half = torch.div(n, 2, rounding_mode="floor")
    s = torch.ldexp(torch.ldexp(b, half.unsqueeze(-1)), (n - half).unsqueeze(-1))
    return c, s.clamp(-6.0, 6.0)


def _index(s):
    """Indices into E2M1 of |s|, to nearest, ties to the even index."""
    a = s.abs()
    return ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int()
            + (a >= 3.5).int() + (a > 5.0).int())


def _round(v):
    """fp32 rows [.., K] (K a multiple of 32) rounded to MXFP4: their values, in fp32."""
    c, s = _blocks(v)
    q = torch.tensor(E2M1, device=v.device)[_index(s)]
    q = torch.where(torch.signbit(s), -q, q)
    n = c - 127
    half = torch.div(n, 2, rounding_mode="floor")
    return torch.ldexp(torch.ldexp(q, half.unsqueeze(-1)), (n - half).unsqueeze(-1)).flatten(-2)


def _pack(v):
    """fp32 rows [R, K] as (codes [R, Kp/2] uint8, scales [Kp/256, R, 2] int32)."""
    R, K = v.shape
    v = torch.nn.functional.pad(v, (0, _padded(K) - K))
    c, s = _blocks(v)
    code = (_index(s) + 8 * torch.signbit(s).int()).flatten(-2).to(torch.uint8)
    codes = code[:, 0::2] | (code[:, 1::2] << 4)
    c = c.to(torch.uint8).view(R, -1, 4, 2).permute(1, 0, 3, 2).contiguous()
    return codes, c.view(torch.int32).squeeze(-1)


def _unpack(codes, scales, K):
    """The fp32 values [R, K] of packed rows."""
    R = codes.shape[0]
    table = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=codes.device)
    q = table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    c = scales.unsqueeze(-1).view(torch.uint8).permute(1, 0, 3, 2).reshape(R, -1)
    return (q.view(R, -1, 32) * torch.exp2(c.float() - 127.0).unsqueeze(-1)).flatten(-2)[:, :K]


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------
def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _routing(shape, T, alpha, g):
    """Routed tokens of a shard: ids [T, k], gate weights, the assignments' rows
    (dest [T * k], -1 where the expert is remote), the rows' assignments
    (perm_src [T * k]) and the offsets of the local experts. The local experts of
    a shard hold one rank of each group of E / E_local consecutive ranks."""
    H, I, E, k, E_local, _ = SHAPES[shape]
    step = E // E_local
    rank = torch.randperm(E, generator=g, device="cuda")
    z = torch.randn((T, E), generator=g, device="cuda") - alpha * torch.log(rank.float() + 1.0)
    top, ids = torch.sort(z, dim=1, descending=True, stable=True)
    top, ids = top[:, :k], ids[:, :k].contiguous()
    by_rank = torch.empty_like(rank)
    by_rank[rank] = torch.arange(E, device="cuda")
    pick = torch.randint(step, (E_local,), generator=g, device="cuda")
    local = by_rank[torch.arange(E_local, device="cuda") * step + pick]
    slot = torch.full((E,), E_local, dtype=torch.int64, device="cuda")
    slot[local] = torch.arange(E_local, device="cuda")
    s = slot[ids].flatten()
    order = torch.sort(s, stable=True)[1]
    counts = torch.bincount(s, minlength=E_local + 1)[:E_local]
    ends = torch.cumsum(counts, 0)
    m = int(ends[-1])
    dest = torch.full((T * k,), -1, dtype=torch.int32, device="cuda")
    dest[order[:m]] = torch.arange(m, dtype=torch.int32, device="cuda")
    offsets = torch.zeros(E_local + 1, dtype=torch.int32, device="cuda")
    offsets[1:] = ends.int()
    return {"ids": ids.int(), "weights": torch.softmax(top, 1).contiguous(), "dest": dest, "perm_src": order.int(),
            "offsets": offsets, "bounds": [0] + ends.tolist(), "m": m, "k": k, "E": E}


def _weights(n, rows, K, g):
    """n matrices [rows, K] of normally distributed weights in MXFP4."""
    codes = torch.empty((n, rows, _padded(K) // 2), dtype=torch.uint8, device="cuda")
    scales = torch.empty((n, _padded(K) // 256, rows, 2), dtype=torch.int32, device="cuda")
    for e in range(n):
        codes[e], scales[e] = _pack(torch.randn((rows, K), generator=g, device="cuda") / math.sqrt(K))
    return {"codes": codes, "scales": scales, "K": K}


def prepare(case, seed):
    g, kind = _gen(seed), case["kind"]
    if kind == "quant":
        # rows of different sizes, as activations and weights have
        x = torch.randn((case["rows"], case["K"]), generator=g, device="cuda")
        x *= torch.exp(torch.randn((case["rows"], 1), generator=g, device="cuda"))
        return {"kind": kind, "x": x if case["dtype"] == "fp32" else x.bfloat16(), "bufs": {}}
    if kind == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        rank = torch.randperm(E, generator=g, device="cuda")
        z = torch.randn((T, E), generator=g, device="cuda") - case["alpha"] * torch.log(rank.float() + 1.0)
        top, ids = torch.sort(z, dim=1, descending=True, stable=True)
        mask = None
        if case["pad"] > 0.0:  # the padding stands at the end of a sequence
            n = case["seq"] or T
            cut = n - torch.randint(int(case["pad"] * n) + 1, (T // n, 1), generator=g, device="cuda")
            mask = (torch.arange(n, device="cuda").unsqueeze(0) < cut).to(torch.uint8).reshape(T)
        return {"kind": kind, "z": z, "ids": ids[:, :k].int().contiguous(), "mask": mask, "seq": case["seq"],
                "weights": torch.softmax(top[:, :k], 1).contiguous(),
                "dweights": torch.randn((T, k), generator=g, device="cuda") / T,
                "dloss": torch.tensor([0.01, 0.001], device="cuda"), "bufs": {}}
    H, I, E, k, E_local, _ = SHAPES[case["shape"]]
    T = case["T"]
    dt = torch.float32 if case["shape"] == "tiny" else torch.bfloat16
    if kind == "router":
        # the gradient of a softmax: rows that sum to nearly nothing, of unequal sizes
        p = torch.softmax(2.0 * torch.randn((T, E), generator=g, device="cuda"), 1)
        dz = p * torch.randn((T, E), generator=g, device="cuda") / T
        return {"kind": kind, "dz": dz - p * dz.sum(1, keepdim=True), "bufs": {},
                "x": torch.randn((T, H), generator=g, device="cuda").to(dt),
                "w": (torch.randn((E, H), generator=g, device="cuda") / math.sqrt(H)).to(dt)}
    s = _routing(case["shape"], T, case["alpha"], g)
    s.update(kind=kind, bufs={}, T=T)
    if kind == "ffn":
        s["x"] = torch.randn((T, H), generator=g, device="cuda").to(dt)
        s["wg"], s["wu"], s["wd"] = _weights(E_local, I, H, g), _weights(E_local, I, H, g), _weights(E_local, H, I, g)
        # room for every assignment; the rows past the routed ones stay as they are
        s["y"] = torch.zeros((T * k, H), dtype=torch.bfloat16, device="cuda")
        return s
    s["dout"] = (torch.randn((T, H), generator=g, device="cuda") / T).to(dt)
    s["y"] = torch.randn((T * k, H), generator=g, device="cuda", dtype=dt)
    s["dy"] = torch.zeros((T * k, H), dtype=dt, device="cuda")
    return s


# ---------------------------------------------------------------------------
# One pass
# ---------------------------------------------------------------------------
def _silu(g):
    return g / (1.0 + torch.exp(-g))


def _plain_ffn(s):
    x = _round(s["x"].float())[(s["perm_src"][: s["m"]] // s["k"]).long()]
    y, b = s["y"], s["bounds"]
    for e in range(len(b) - 1):  # the experts' row counts differ: a product of their own for each
        if b[e] == b[e + 1]:
            continue
        wg, wu, wd = (_unpack(w["codes"][e], w["scales"][e], w["K"]) for w in (s["wg"], s["wu"], s["wd"]))
        r = x[b[e]:b[e + 1]]
        h = _round(_silu(r @ wg.t()) * (r @ wu.t()))
        y[b[e]:b[e + 1]] = (h @ wd.t()).bfloat16()
    return y


def _plain_balance(s):
    z, ids, k = s["z"], s["ids"], s["ids"].shape[1]
    T, E = z.shape
    n = s["seq"] or T
    S = T // n
    live = torch.ones(T, device=z.device) if s["mask"] is None else (s["mask"] != 0).float()
    top = z.amax(1, keepdim=True)
    ex = torch.exp(z - top)
    total = ex.sum(1, keepdim=True)
    p, lse = ex / total, top + torch.log(total)
    hit = (ids.unsqueeze(2) == torch.arange(E, device=z.device, dtype=torch.int32)).float()  # [T, k, E]
    counts = (hit.sum(1) * live.unsqueeze(1)).view(S, n, E).sum(1)
    tokens = live.view(S, n).sum(1)
    P = (p * live.unsqueeze(1)).view(S, n, E).sum(1)
    factor = torch.where(tokens > 0, E / (k * tokens * tokens).clamp(min=1.0), torch.zeros_like(tokens))
    factor = factor / (tokens > 0).sum().clamp(min=1)
    many = live.sum().clamp(min=1.0)
    loss = torch.stack(((factor * (counts * P).sum(1)).sum(), (live.unsqueeze(1) * lse * lse).sum() / many))
    c = (counts * factor.unsqueeze(1)).repeat_interleave(n, 0)
    dz = s["dloss"][0] * p * (c - (c * p).sum(1, keepdim=True)) + s["dloss"][1] * 2.0 / many * lse * p
    dz = dz * live.unsqueeze(1)
    w, dw = s["weights"], s["dweights"]
    dz = dz + ((w * (dw - (w * dw).sum(1, keepdim=True))).unsqueeze(2) * hit).sum(1)
    return {"loss": loss, "counts": counts.int(), "dlogits": dz}


def _plain_combine(s):
    dest = s["dest"].view(-1, s["k"]).long()
    here = dest >= 0
    do = s["dout"].float()
    rows = s["y"].float()[dest.clamp(min=0)]  # [T, k, H]
    dw = torch.where(here, torch.matmul(rows, do.unsqueeze(2)).squeeze(2), torch.zeros_like(s["weights"]))
    src = s["perm_src"][: s["m"]].long()
    s["dy"][: s["m"]] = (s["weights"].flatten()[src].unsqueeze(1) * do[src // s["k"]]).to(s["dout"].dtype)
    return {"dweights": dw, "dy": s["dy"]}


def _plain(s):
    kind = s["kind"]
    if kind == "quant":
        return _round(s["x"].float()).bfloat16()
    if kind == "ffn":
        return _plain_ffn(s)
    if kind == "balance":
        return _plain_balance(s)
    if kind == "combine":
        return _plain_combine(s)
    x, dz = s["x"].float(), s["dz"]
    return {"dx": (dz @ s["w"].float()).to(s["x"].dtype), "dw": dz.t() @ x, "dbias": dz.sum(0)}


def _own(s):
    import paper_2606_00735_amd as moe

    kind, b = s["kind"], s["bufs"]  # b: what a program keeps between passes
    if kind == "quant":
        b["q"] = moe.moe_mx4_quantize(s["x"], out=b.get("q"))
        b["v"] = moe.moe_mx4_dequantize(b["q"], out=b.get("v"))
        return b["v"]
    if kind == "ffn":
        w = [moe.Mx4Tensor(m["codes"], m["scales"], m["K"]) for m in (s["wg"], s["wu"], s["wd"])]
        b["x"] = moe.moe_mx4_quantize(s["x"], out=b.get("x"))
        y, b["ws"] = moe.moe_grouped_swiglu_ffn_mx4(b["x"], *w, s["offsets"], perm_src=s["perm_src"], k=s["k"],
                                                    experts=s["E"], ws=b.get("ws"), y_perm=s["y"])
        return y
    if kind == "balance":
        loss, counts, live, b["ws"] = moe.moe_balance_loss(s["z"], s["ids"], mask=s["mask"], seq_len=s["seq"], ws=b.get("ws"))
        dz = moe.moe_gate_backward(s["z"], s["ids"], counts, live, s["dloss"], weights=s["weights"],
                                   dweights=s["dweights"], mask=s["mask"], seq_len=s["seq"])
        return {"loss": loss, "counts": counts, "dlogits": dz}
    if kind == "combine":
        dw, dy = moe.moe_combine_backward(s["dout"], s["y"], s["weights"], s["dest"], dy_perm=s["dy"])
        return {"dweights": dw, "dy": dy}
    dx, dw, dbias, b["ws"] = moe.moe_router_grad(s["dz"], s["x"], s["w"], ws=b.get("ws"))
    return {"dx": dx, "dw": dw, "dbias": dbias}


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# Work, 64-bit results
# ---------------------------------------------------------------------------
def _routed(shape, T, alpha):
    """Expected rows and active experts of the local share."""
    _, _, E, k, E_local, _ = SHAPES[shape]
    g = torch.Generator()
    g.manual_seed(1)
    z = torch.randn((512, E), generator=g) - alpha * torch.log(torch.arange(E) + 1.0)
    share = torch.bincount(torch.topk(z, k, dim=1)[1].flatten(), minlength=E).double() / 512.0
    mid = share.view(E_local, -1).mean(1).clamp(max=1.0)  # the expected local expert of each group of ranks
    return float(mid.sum()) * T, float((1.0 - (1.0 - mid) ** T).sum())


def work(case):
    kind = case["kind"]
    if kind == "quant":
        n = float(case["rows"] * case["K"])
        # x read, codes and scales written, values written
        return {"bytes": n * ((4 if case["dtype"] == "fp32" else 2) + 17 / 32 + 2), "flops": 4.0 * n}
    if kind == "balance":
        T, E, k = case["T"], case["E"], case["k"]
        # logits read, their gradient written; ids, weights and the weights' gradient
        return {"bytes": 8.0 * T * E + 12.0 * T * k, "flops": 12.0 * T * E}
    H, I, E, k, E_local, _ = SHAPES[case["shape"]]
    T, es = case["T"], 4 if case["shape"] == "tiny" else 2
    if kind == "router":
        return {"bytes": 2.0 * T * H * es + 4.0 * T * E + E * H * (es + 4.0), "flops": 4.0 * T * E * H}
    rows, active = _routed(case["shape"], T, case["alpha"])
    if kind == "combine":
        return {"bytes": es * H * (T + 2.0 * rows) + 12.0 * T * k, "flops": 3.0 * rows * H}
    return {"bytes": 3.0 * H * I * active * 17 / 32 + 2.0 * T * H + 2.0 * rows * H + 4.0 * rows, "flops": 6.0 * H * I * rows}


def _round64(v):
    """Rows rounded to MXFP4 in 64 bits, element by element from the grid's spacing."""
    b = v.unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    e = torch.where(top > 0, torch.floor(torch.log2(torch.where(top > 0, top, 1.0))), torch.full_like(top, -125.0))
    # log2 may round up to a whole number just below a power of two
    e = torch.where(torch.exp2(e) > top, e - 1.0, e)
    s = torch.exp2((e - 2.0).clamp(min=-127.0))
    t = (b / s).clamp(-6.0, 6.0)
    step = torch.where(t.abs() >= 4.0, 2.0, torch.where(t.abs() >= 2.0, 1.0, 0.5)).to(v.dtype)
    return (torch.round(t / step) * step * s).flatten(-2)


def _values64(w, e):
    c = w["codes"][e].long()
    n = torch.stack((c % 16, c // 16), -1).flatten(-2)
    mag, x = n % 2, (n // 2) % 4
    v = torch.where(x == 0, 0.5 * mag, (1.0 + 0.5 * mag) * torch.exp2(x.double() - 1.0)) * (1 - 2 * (n // 8))
    words = w["scales"][e].long() & 0xFFFFFFFF  # [chunk, row, half]
    blocks = [(words[..., b % 2] >> (8 * (b // 2))) & 255 for b in range(8)]
    c = torch.stack(blocks, -1).transpose(0, 1).flatten(1)
    return (v * torch.exp2(c.double() - 127.0).repeat_interleave(32, 1))[:, : w["K"]]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quant":
        return _round64(s["x"].double())
    if kind == "ffn":
        x = _round64(s["x"].double())
        b = s["bounds"]
        y = torch.zeros(s["y"].shape, dtype=torch.float64, device=x.device)
        for e in range(len(b) - 1):
            if b[e] < b[e + 1]:
                r = x[(s["perm_src"][b[e]:b[e + 1]] // s["k"]).long()]
                g = r @ _values64(s["wg"], e).t()
                h = _round64(g * torch.sigmoid(g) * (r @ _values64(s["wu"], e).t()))
                y[b[e]:b[e + 1]] = h @ _values64(s["wd"], e).t()
        return y
    if kind == "balance":
        z, ids = s["z"].double(), s["ids"].long()
        T, E = z.shape
        k, n = ids.shape[1], case["seq"] or T
        live = torch.ones(T, dtype=torch.bool, device=z.device) if s["mask"] is None else s["mask"].bool()
        p, lse = torch.softmax(z, 1), torch.logsumexp(z, 1)
        counts = torch.zeros((T // n, E), dtype=torch.int64, device=z.device)
        balance, dz = [], torch.zeros_like(z)
        for q in range(T // n):
            at = torch.arange(q * n, (q + 1) * n, device=z.device)
            at = at[live[at]]
            if at.numel() == 0:
                continue
            counts[q] = torch.bincount(ids[at].flatten(), minlength=E)
            f = counts[q].double() * E / (k * at.numel())
            balance.append((f * p[at].mean(0)).sum())
            dz[at] = p[at] * (f - (p[at] @ f).unsqueeze(1)) / at.numel()
        many = max(1, int(live.sum()))
        dz *= s["dloss"][0].double() / max(1, len(balance))
        dz[live] += s["dloss"][1].double() * (2.0 / many * lse[live]).unsqueeze(1) * p[live]
        w, dw = s["weights"].double(), s["dweights"].double()
        dz.scatter_add_(1, ids, w * (dw - (w * dw).sum(1, keepdim=True)))
        zero = torch.zeros((), dtype=torch.float64, device=z.device)
        loss = torch.stack((torch.stack(balance).mean() if balance else zero, (lse[live] ** 2).sum() / many))
        return {"loss": loss, "counts": counts.int(), "dlogits": dz}
    if kind == "combine":
        k, do = s["k"], s["dout"].double()
        src = s["perm_src"][: s["m"]].long()
        y, tok = s["y"][: s["m"]].double(), src // k
        dw = torch.zeros(s["dest"].numel(), dtype=torch.float64, device=do.device)
        dw[src] = (y * do[tok]).sum(1)
        dy = torch.zeros(s["dy"].shape, dtype=torch.float64, device=do.device)
        dy[: s["m"]] = s["weights"].double().flatten()[src].unsqueeze(1) * do[tok]
        return {"dweights": dw.view(-1, k), "dy": dy}
    dz, x = s["dz"].double(), s["x"].double()
    return {"dx": dz @ s["w"].double(), "dw": dz.t() @ x, "dbias": dz.sum(0)}

