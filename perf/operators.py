"""The operators of an attention layer around the banded attention, as cases that can be timed and compared: layer norm
and its gradient, rotary positions and their gradient, softmax attention on a band and its gradient.

`listed()` names the cases that are quoted, `draw(rng)` gives another one of the same ranges, `prepare(case, seed)` makes
what a program holds before the call, `run(state)` is one pass, `work(case)` what the pass cannot do without and
`exact(case, seed)` the outputs in 64 bits.  `own` chooses between the library's calls and elementary torch operations.

Fields of a case:
  op      "layer_norm_fwd", "layer_norm_bwd"   rows, D, dtype, wdtype, residual
          "rope_fwd", "rope_bwd"               B, Hq, Hk, L, d, rot, interleaved, scaling, factor, positions, layout, dtype
          "attn_fwd", "attn_bwd"               B, Hq, Hk, Lq, Lk, d, W, causal, eps, kind, layout, dtype
  positions  "zero" (token l at position l), "start" (from a position per item on), "each" (a position per token)
  kind       "plain"; "varlen" (padded batch); "masked" (inactive tokens too); "cached" (the Lq last tokens of ragged caches)
  layout     "bhld" (contiguous heads), "blhd" (the heads of a token adjacent, as a projection leaves them)
"""
import math

import torch

own = False
EPS = 1e-5   # under layer norm's root
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def _norm(name, op, rows, D, dtype, wdtype, residual):
    return {"name": name, "op": op, "rows": rows, "D": D, "dtype": dtype, "wdtype": wdtype, "residual": residual}


def _rope(name, op, B, Hq, Hk, L, d, rot, interleaved, scaling, factor, positions, layout, dtype):
    return {"name": name, "op": op, "B": B, "Hq": Hq, "Hk": Hk, "L": L, "d": d, "rot": rot, "interleaved": interleaved,
            "scaling": scaling, "factor": factor, "positions": positions, "layout": layout, "dtype": dtype}


def _attn(name, op, B, Hq, Hk, Lq, Lk, d, W, causal, eps, kind, layout, dtype):
    return {"name": name, "op": op, "B": B, "Hq": Hq, "Hk": Hk, "Lq": Lq, "Lk": Lk, "d": d, "W": W, "causal": causal,
            "eps": eps, "kind": kind, "layout": layout, "dtype": dtype}


def listed():
    return [
        # the smallest configuration's tokens, fp32: launches and latency
        _norm("norm_short", "layer_norm_fwd", 256, 128, "f32", "f32", False),
        # the norm in front of a layer on the longest context, with the residual sum that it takes on
        _norm("norm_long", "layer_norm_fwd", 262144, 512, "bf16", "f32", True),
        # training of a small model, 4 sequences of 4096 tokens, 8 heads of 64
        _norm("norm_grad", "layer_norm_bwd", 16384, 512, "bf16", "f32", True),
        # fp32 and a width and a number of rows that fit no vector and no tile
        _norm("norm_grad_odd", "layer_norm_bwd", 30011, 1283, "f32", "f32", False),
        # the newest token of 8 sequences, far along a scaled context
        _rope("rope_token", "rope_fwd", 8, 8, 2, 1, 64, 64, False, "yarn", 8.0, "start", "blhd", "bf16"),
        # the longest context, from the projections' layout into the one that the banded attention reads
        _rope("rope_long", "rope_fwd", 1, 2, 2, 262144, 64, 64, False, "yarn", 8.0, "zero", "blhd", "bf16"),
        # gradients in fp32, half of a wide head turned, adjacent pairs, packed sequences
        _rope("rope_grad", "rope_bwd", 2, 8, 4, 3001, 128, 64, True, "none", 1.0, "each", "bhld", "f32"),
        # answering: one token of each of 4 sequences against ragged caches
        _attn("attn_token", "attn_fwd", 4, 8, 2, 1, 65536, 64, 1 << 20, True, 1.0, "cached", "bhld", "bf16"),
        # forward on the longest context and its band (benchmark configuration)
        _attn("attn_paper", "attn_fwd", 1, 2, 2, 262144, 262144, 64, 256, False, 0.5, "plain", "bhld", "bf16"),
        # gradient check at an ordinary size: fp32, padded batch with inactive tokens, rows that are left empty
        _attn("attn_grad_masked", "attn_bwd", 2, 4, 4, 701, 701, 32, 64, False, 1.0, "masked", "bhld", "f32"),
        # training with shared, wide heads over everything before a token
        _attn("attn_grad_dense", "attn_bwd", 1, 16, 4, 4096, 4096, 128, 4096, True, 1.0, "plain", "blhd", "bf16"),
        # the gradient on the longest context (benchmark configuration)
        _attn("attn_grad_paper", "attn_bwd", 1, 2, 2, 262144, 262144, 64, 256, False, 0.5, "plain", "bhld", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _edges(c):
    """Expected pairs of a query and a key for one query head of the whole batch."""
    full = 0.75 if c["kind"] != "plain" else 1.0
    Lk = c["Lk"] * full
    p = torch.arange(c["Lq"], dtype=torch.float64) + (max(Lk - c["Lq"], 0) if c["kind"] == "cached" else 0)
    hi = torch.clamp(p if c["causal"] else p + c["W"], max=Lk - 1)
    lo = torch.clamp(p - c["W"], min=0)
    n = float(torch.clamp(hi - lo + 1, min=0).sum()) * c["B"]
    if c["kind"] in ("varlen", "masked"):
        n *= full
    return n * (0.8 if c["kind"] == "masked" else 1.0)


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"].startswith("layer_norm"):
        n, fwd = case["rows"] * case["D"], case["op"].endswith("fwd")
        return {"bytes": n * e * ((2 if fwd else 3) + (2 if fwd else 1) * case["residual"]) + 8 * case["rows"], "flops": (8 if fwd else 14) * n}
    if case["op"].startswith("rope"):
        n = case["B"] * case["L"] * (case["Hq"] + case["Hk"])
        return {"bytes": 2 * n * case["d"] * e, "flops": 3 * n * case["rot"]}
    B, d, q, k = case["B"], case["d"], case["Hq"] * case["Lq"], case["Hk"] * case["Lk"]
    if case["kind"] == "cached":   # of a cache only what a token reaches
        k = case["Hk"] * min(0.75 * case["Lk"], case["Lq"] + (1 if case["causal"] else 2) * case["W"])
    edges = _edges(case) * case["Hq"]
    if case["op"] == "attn_fwd":
        return {"bytes": B * (2 * q * d * e + 4 * q + 2 * k * d * e), "flops": 4 * d * edges}
    return {"bytes": B * (4 * q * d * e + 4 * q + 4 * k * d * e), "flops": 10 * d * edges}


def _draw(rng):
    op = rng.choice(["layer_norm_fwd", "layer_norm_bwd", "rope_fwd", "rope_bwd", "attn_fwd", "attn_fwd", "attn_bwd", "attn_bwd"])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    if op.startswith("layer_norm"):
        D = rng.choice([64 * rng.randint(1, 32), 8 * _log(rng, 4, 500), _log(rng, 17, 5000)])
        return _norm("", op, _log(rng, 1, 262144), D, dtype, rng.choice([dtype, "f32"]), rng.random() < 0.5)
    Hk = rng.choice([1, 2, 4])
    Hq, d = Hk * rng.choice([1, 1, 2, 3, 4]), rng.choice([32, 64, 64, 128])
    layout, B = rng.choice(["bhld", "blhd"]), rng.choice([1, 1, 2, 3, 4])
    if op.startswith("rope"):
        return _rope("", op, B, Hq, Hk, _log(rng, 1, 262144), d, rng.choice([d, d, d // 2, d // 4 + 2]), rng.random() < 0.5,
                     rng.choice(["none", "linear", "ntk", "yarn"]), rng.choice([1.5, 4.0, 8.0]),
                     rng.choice(["zero", "start", "each"]), layout, dtype)
    eps, causal = rng.choice([0.5, 1.0]), rng.random() < 0.5
    if op == "attn_fwd" and rng.random() < 0.4:
        Lk = _log(rng, 64, 131072)
        return _attn("", op, B, Hq, Hk, min(Lk, rng.choice([1, 1, 2, 5, 17])), Lk, d, rng.choice([1 << 20, 1 << 20, _log(rng, 16, 4096)]),
                     True, eps, "cached", layout, dtype)
    if rng.random() < 0.5:   # a band on long sequences
        L = _log(rng, 300, 262144)
        W = _log(rng, 1, 1024)
    else:                    # everything, on short ones
        L = _log(rng, 1, 4096)
        W = L
    return _attn("", op, B, Hq, Hk, L, L, d, W, causal, eps, rng.choice(["plain", "plain", "varlen", "masked"]), layout, dtype)


def _cost(c):
    """Seconds at round rates of the bytes and of the products, the latter weighted by the type."""
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if c["dtype"] == "bf16" else 1e14)) + w["bytes"] / 1e15


def draw(rng):
    """A case of the ranges above that costs no more than the largest listed one, of plain and of library operations."""
    most = max(_cost(c) for c in listed())
    wide = max(_plain_pairs(c) for c in listed() if c["op"].startswith("attn"))
    while True:
        c = _draw(rng)
        if _cost(c) <= most and (not c["op"].startswith("attn") or _plain_pairs(c) <= wide):
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------------ inputs
def frequencies(rot, base, scaling, factor, trained):
    """Radians per position of each pair, float64, and the factor that turned features are multiplied by."""
    k = torch.arange(rot // 2, dtype=torch.float64)
    freq, amplitude = base ** (-2.0 * k / rot), 1.0
    if scaling == "linear":      # positions divided by the factor
        freq = freq / factor
    elif scaling == "ntk":       # a larger base: the slowest pair by the factor, the fastest not at all
        freq = (base * factor ** (rot / max(rot - 2, 1))) ** (-2.0 * k / rot)
    elif scaling == "yarn":      # pairs that turn often within the trained length as they are, those that hardly do divided:
        # the pair index at which a pair turns 32 times, and once, within it
        at = [rot * math.log(trained / (n * 2 * math.pi)) / (2 * math.log(base)) for n in (32.0, 1.0)]
        lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), rot - 1)
        ramp = ((k - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        freq = freq * (1 - ramp) + freq / factor * ramp
        amplitude = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    return freq, amplitude


def _heads(g, B, H, L, d, c):
    shape = (B, L, H, d) if c["layout"] == "blhd" else (B, H, L, d)
    x = torch.randn(shape, generator=g, device="cuda").to(DTYPES[c["dtype"]])
    return x.transpose(1, 2) if c["layout"] == "blhd" else x


def _lens(g, B, L):
    return torch.randint((L + 1) // 2, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    s = {"case": c}
    if c["op"].startswith("layer_norm"):
        n, D, wt = c["rows"], c["D"], DTYPES[c["wdtype"]]
        # activations with a mean of their own and some features that are larger throughout
        big = 1 + 4 * (torch.rand(D, generator=g, device="cuda") > 0.97).float()
        make = lambda: ((torch.randn((n, D), generator=g, device="cuda") * big + 0.3)).to(dt)   # noqa: E731
        s["x"] = make()
        s["w"] = (1 + 0.2 * torch.randn(D, generator=g, device="cuda")).to(wt)
        s["b"] = (0.1 * torch.randn(D, generator=g, device="cuda")).to(wt)
        s["r"] = make() if c["residual"] and c["op"] == "layer_norm_fwd" else None
        if c["op"] == "layer_norm_bwd":
            s["dy"] = torch.randn((n, D), generator=g, device="cuda").to(dt)
            s["ds"] = torch.randn((n, D), generator=g, device="cuda").to(dt) if c["residual"] else None
            x = s["x"].double()
            s["stats"] = torch.stack([x.mean(1), (x.var(1, unbiased=False) + EPS).rsqrt()]).float()
        return s
    B = c["B"]
    if c["op"].startswith("rope"):
        s["q"], s["k"] = _heads(g, B, c["Hq"], c["L"], c["d"], c), _heads(g, B, c["Hk"], c["L"], c["d"], c)
        freq, s["amplitude"] = frequencies(c["rot"], 10000.0, c["scaling"], c["factor"], 32768)
        s["freq"] = freq.cuda()
        s["start"] = torch.randint(0, 200000, (B,), generator=g, device="cuda", dtype=torch.int32) if c["positions"] == "start" else None
        s["pos"] = torch.randint(0, 262144, (B, c["L"]), generator=g, device="cuda", dtype=torch.int32) if c["positions"] == "each" else None
        return s
    s["q"] = _heads(g, B, c["Hq"], c["Lq"], c["d"], c)
    s["k"], s["v"] = _heads(g, B, c["Hk"], c["Lk"], c["d"], c), _heads(g, B, c["Hk"], c["Lk"], c["d"], c)
    s["len_q"] = s["len_k"] = s["mask_q"] = s["mask_k"] = s["start"] = None
    if c["kind"] == "cached":
        s["len_k"] = torch.clamp(_lens(g, B, c["Lk"]), min=c["Lq"])
        s["start"] = s["len_k"] - c["Lq"]
    elif c["kind"] != "plain":
        s["len_q"], s["len_k"] = _lens(g, B, c["Lq"]), _lens(g, B, c["Lk"])
    if c["kind"] == "masked":
        # runs of inactive tokens, some longer than a narrow band
        s["mask_q"], s["mask_k"] = ((torch.rand((B, (n + 15) // 16), generator=g, device="cuda") > 0.2).repeat_interleave(16, 1)[:, :n].to(torch.uint8).contiguous()
                                    for n in (c["Lq"], c["Lk"]))
    if c["op"] == "attn_bwd":
        s["do"] = _heads(g, B, c["Hq"], c["Lq"], c["d"], c)
        o, s["lse"] = _plain_attn_fwd(s)
        s["o"] = torch.empty_like(s["q"]).copy_(o)
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_norm_fwd(s):
    r = s["r"]
    x = s["x"] if r is None else (s["x"].float() + r.float()).to(s["x"].dtype)
    f = x.float()
    mean = f.mean(1, keepdim=True)
    rstd = ((f - mean).square().mean(1, keepdim=True) + EPS).rsqrt()
    y = ((f - mean) * rstd * s["w"].float() + s["b"].float()).to(x.dtype)
    return y, x, torch.stack([mean[:, 0], rstd[:, 0]])


def _plain_norm_bwd(s):
    dy, w = s["dy"].float(), s["w"]
    mean, rstd = s["stats"][0][:, None], s["stats"][1][:, None]
    xh = (s["x"].float() - mean) * rstd
    gy = dy * w.float()
    dx = rstd * (gy - gy.mean(1, keepdim=True) - xh * (gy * xh).mean(1, keepdim=True))
    if s["ds"] is not None:
        dx = dx + s["ds"].float()
    return dx.to(s["x"].dtype), (dy * xh).sum(0).to(w.dtype), dy.sum(0).to(w.dtype)


def _plain_rope(s, back):
    c = s["case"]
    pos = torch.arange(c["L"], device="cuda")[None]
    if s["start"] is not None:
        pos = pos + s["start"].long()[:, None]
    if s["pos"] is not None:
        pos = s["pos"]
    theta = pos.double()[:, None, :, None] * s["freq"]
    cos, sin = (theta.cos() * s["amplitude"]).float(), (theta.sin() * s["amplitude"]).float()
    return _turn(s["q"], cos, -sin if back else sin, c), _turn(s["k"], cos, -sin if back else sin, c)


def _turn(x, cos, sin, c):
    f, h = x.float(), c["rot"] // 2
    a, b = (f[..., 0:2 * h:2], f[..., 1:2 * h:2]) if c["interleaved"] else (f[..., :h], f[..., h:2 * h])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, f[..., 2 * h:]], -1).to(x.dtype).contiguous()


def _rows(c):
    """Query rows that share one window of keys, and the window's keys."""
    C = c["Lq"] if 2 * c["W"] + 1 >= c["Lk"] or c["Lq"] <= 64 else min(c["Lq"], max(64, c["W"]))
    return C, min(c["Lk"], C + 2 * c["W"])


def _plain_pairs(c):
    C, m = _rows(c)
    return c["B"] * c["Hq"] * -(-c["Lq"] // C) * C * m * (1 if c["op"] == "attn_fwd" else 2)


def _windows(s):
    """Queries [B, Hk, n, G C, d], keys and values [B, Hk, n, m, d] of n chunks of C query rows, the keys' indices and which pairs count."""
    c = s["case"]
    C, m = _rows(c)
    n, G, Lq, Lk, B, Hk, d, W = -(-c["Lq"] // C), c["Hq"] // c["Hk"], c["Lq"], c["Lk"], c["B"], c["Hk"], c["d"], c["W"]
    dev = "cuda"
    start = torch.zeros(B, dtype=torch.long, device=dev) if s["start"] is None else s["start"].long()
    i = torch.arange(n * C, device=dev).view(1, n, C)
    p = i + start[:, None, None]                                                    # [B, n, C] positions
    at = (p[:, :, :1] - W).clamp(0, Lk - m) + torch.arange(m, device=dev)           # [B, n, m] keys
    rows = torch.full((B,), Lq, device=dev) if s["len_q"] is None else s["len_q"].long()
    keys = torch.full((B,), Lk, device=dev) if s["len_k"] is None else s["len_k"].long()
    row_ok, key_ok = (i < rows[:, None, None]).expand(B, n, C), at < keys[:, None, None]
    if s["mask_q"] is not None:
        row_ok = row_ok & (s["mask_q"].bool()[:, i.view(-1).clamp(max=Lq - 1)].view(B, n, C))
    if s["mask_k"] is not None:
        key_ok = key_ok & s["mask_k"].bool().gather(1, at.view(B, -1)).view(B, n, m)
    gap = at[:, :, None, :] - p[..., None]
    ok = (gap.abs() <= W) & row_ok[..., None] & key_ok[:, :, None, :]
    if c["causal"]:
        ok = ok & (gap <= 0)
    ok = ok[:, None, :, None].expand(B, 1, n, G, C, m).reshape(B, 1, n, G * C, m)
    # [B, n, m, Hk, d] by index, heads in front
    pick = lambda x: x.transpose(1, 2)[torch.arange(B, device=dev)[:, None, None], at].permute(0, 3, 1, 2, 4).float().contiguous()   # noqa: E731
    return pick(s["k"]), pick(s["v"]), at, ok, (C, m, n, G)


def _chunks(x, C, n, G):
    """[B, Hq, Lq, d] -> [B, Hk, n, G C, d] in fp32, rows beyond Lq zero."""
    B, Hq, Lq, d = x.shape
    f = torch.zeros((B, Hq, n * C, d), device="cuda", dtype=torch.float32)
    f[:, :, :Lq] = x.float()
    return f.view(B, Hq // G, G, n, C, d).transpose(2, 3).reshape(B, Hq // G, n, G * C, d)


def _unchunk(x, C, n, G, Lq):
    B, Hk = x.shape[:2]
    return x.view(B, Hk, n, G, C, -1).transpose(2, 3).reshape(B, Hk * G, n * C, -1)[:, :, :Lq]


def _plain_attn_fwd(s):
    c = s["case"]
    k, v, _, ok, (C, m, n, G) = _windows(s)
    score = torch.matmul(_chunks(s["q"], C, n, G), k.transpose(-1, -2)) * (1.0 / (c["eps"] * math.sqrt(c["d"])))
    score = score.masked_fill(~ok, -math.inf)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - top.clamp(min=-3e38))
    total = e.sum(-1, keepdim=True)
    o = torch.matmul(e, v) / torch.where(total > 0, total, 1.0)
    return _unchunk(o, C, n, G, c["Lq"]).to(s["q"].dtype), _unchunk(top + total.log(), C, n, G, c["Lq"])[..., 0].contiguous()


def _plain_attn_bwd(s):
    c = s["case"]
    scale = 1.0 / (c["eps"] * math.sqrt(c["d"]))
    k, v, at, ok, (C, m, n, G) = _windows(s)
    q, o, do = (_chunks(s[x], C, n, G) for x in ("q", "o", "do"))
    lse = _chunks(torch.where(s["lse"] > -math.inf, s["lse"], 0.0)[..., None], C, n, G)
    p = torch.exp((torch.matmul(q, k.transpose(-1, -2)) * scale - lse).masked_fill(~ok, -math.inf))
    dv = torch.matmul(p.transpose(-1, -2), do)
    ds = p * (torch.matmul(do, v.transpose(-1, -2)) - (do * o).sum(-1, keepdim=True)) * scale
    dq = _unchunk(torch.matmul(ds, k), C, n, G, c["Lq"])
    dk = torch.matmul(ds.transpose(-1, -2), q)

    def gather(x):   # [B, Hk, n, m, d] -> [B, Hk, Lk, d], windows overlap
        B, Hk, d = c["B"], c["Hk"], c["d"]
        out = torch.zeros((B * c["Lk"], Hk, d), device="cuda", dtype=torch.float32)
        index = (at + torch.arange(B, device="cuda")[:, None, None] * c["Lk"]).view(-1)
        out.index_add_(0, index, x.permute(0, 2, 3, 1, 4).reshape(-1, Hk, d))
        return out.view(B, c["Lk"], Hk, d).transpose(1, 2).to(s["k"].dtype)

    return dq.to(s["q"].dtype), gather(dk), gather(dv)


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    s = state
    c = s["case"]
    op = c["op"]
    if own:
        import paper_2605_08123_amd as ska
        if op == "layer_norm_fwd":
            return ska.ska_layer_norm_fwd(s["x"], s["w"], s["b"], residual=s["r"], eps=EPS)
        if op == "layer_norm_bwd":
            return ska.ska_layer_norm_bwd(s["dy"], s["x"], s["w"], s["stats"], dS=s["ds"])
        if op == "rope_fwd":
            return ska.ska_rope_fwd(s["q"], s["k"], s["freq"], amplitude=s["amplitude"], interleaved=c["interleaved"],
                                    start=s["start"], positions=s["pos"])
        if op == "rope_bwd":
            return ska.ska_rope_bwd(s["q"], s["k"], s["freq"], amplitude=s["amplitude"], interleaved=c["interleaved"],
                                    start=s["start"], positions=s["pos"])
        where = dict(causal=c["causal"], eps=c["eps"], len_q=s["len_q"], len_k=s["len_k"], mask_q=s["mask_q"],
                     mask_k=s["mask_k"], start_q=s["start"])
        if op == "attn_fwd":
            return ska.ska_softmax_attn_fwd(s["q"], s["k"], s["v"], c["W"], **where)
        return ska.ska_softmax_attn_bwd(s["q"], s["k"], s["v"], s["o"], s["do"], s["lse"], c["W"], **where)
    if op == "layer_norm_fwd":
        return _plain_norm_fwd(s)
    if op == "layer_norm_bwd":
        return _plain_norm_bwd(s)
    if op.startswith("rope"):
        return _plain_rope(s, op == "rope_bwd")
    return _plain_attn_fwd(s) if op == "attn_fwd" else _plain_attn_bwd(s)


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "layer_norm_fwd":
        x = s["x"] if s["r"] is None else (s["x"].double() + s["r"].double()).to(s["x"].dtype)   # the sum as it is stored
        f = x.double()
        var, mean = torch.var_mean(f, dim=1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        return torch.addcmul(s["b"].double(), (f - mean[:, None]) / torch.sqrt(var + EPS)[:, None], s["w"].double()), x, torch.stack([mean, rstd])
    if c["op"] == "layer_norm_bwd":
        x, w = s["x"].double().requires_grad_(), s["w"].double().requires_grad_()
        b = torch.zeros_like(w).requires_grad_()
        var, mean = torch.var_mean(x, dim=1, correction=0)
        y = (x - mean[:, None]) / torch.sqrt(var + EPS)[:, None] * w + b
        loss = (y * s["dy"].double()).sum()
        if s["ds"] is not None:
            loss = loss + (x * s["ds"].double()).sum()
        return torch.autograd.grad(loss, (x, w, b))
    if c["op"].startswith("rope"):
        pos = torch.arange(c["L"], device="cuda").expand(c["B"], -1)
        if s["start"] is not None:
            pos = pos + s["start"][:, None]
        if s["pos"] is not None:
            pos = s["pos"]
        angle = pos.double()[..., None] * s["freq"] * (-1 if c["op"] == "rope_bwd" else 1)
        unit = torch.polar(torch.full_like(angle, s["amplitude"]), angle)[:, None]
        outs = []
        for x in (s["q"], s["k"]):
            f, h = x.double(), c["rot"] // 2
            part = f[..., :2 * h].unflatten(-1, (h, 2)) if c["interleaved"] else f[..., :2 * h].unflatten(-1, (2, h)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(part.contiguous()) * unit)
            z = z.flatten(-2) if c["interleaved"] else z.transpose(-1, -2).flatten(-2)
            outs.append(torch.cat([z, f[..., 2 * h:]], -1))
        return tuple(outs)
    return _exact_attn(s)


def _exact_attn(s):
    """By the definition, a piece of the query rows after another; gradients by differentiating it."""
    c = s["case"]
    B, Hq, Hk, Lq, Lk, W = (c[x] for x in ("B", "Hq", "Hk", "Lq", "Lk", "W"))
    G, back = Hq // Hk, c["op"] == "attn_bwd"
    out = torch.zeros((B, Hq, Lq, c["d"]), device="cuda", dtype=torch.float64)
    lse = torch.full((B, Hq, Lq), -math.inf, device="cuda", dtype=torch.float64)
    dk, dv = (torch.zeros((B, Hk, Lk, c["d"]), device="cuda", dtype=torch.float64) for _ in range(2))
    step = 2048 if W < Lk else 512
    ints = lambda x, other: [other] * B if x is None else x.tolist()   # noqa: E731
    lens_q, lens_k, starts = ints(s["len_q"], Lq), ints(s["len_k"], Lk), ints(s["start"], 0)
    for b in range(B):
        for i0 in range(0, lens_q[b], step):
            i1 = min(lens_q[b], i0 + step)
            j0, j1 = max(0, i0 + starts[b] - W), min(lens_k[b], i1 + starts[b] + (0 if c["causal"] else W))
            if j0 >= j1:
                continue
            p, j = torch.arange(i0, i1, device="cuda")[:, None] + starts[b], torch.arange(j0, j1, device="cuda")
            off = (j > p + W) | (j < p - W)
            if c["causal"]:
                off = off | (j > p)
            if s["mask_q"] is not None:
                off = off | (s["mask_q"][b, i0:i1, None] == 0)
            if s["mask_k"] is not None:
                off = off | (s["mask_k"][b, j0:j1] == 0)
            q = s["q"][b, :, i0:i1].double().unflatten(0, (Hk, G)).requires_grad_(back)
            k, v = (s[x][b, :, None, j0:j1].double().requires_grad_(back) for x in ("k", "v"))
            a = (q @ k.transpose(-1, -2)) / (c["eps"] * c["d"] ** 0.5)
            a = torch.where(off, -1e300, a)
            top = a.detach().amax(-1, keepdim=True)
            e = torch.where(off, 0.0, torch.exp(a - top))
            total = e.sum(-1, keepdim=True)
            o = (e @ v) / torch.where(total == 0, 1.0, total)
            if back:
                gq, gk, gv = torch.autograd.grad(o, (q, k, v), s["do"][b, :, i0:i1].double().unflatten(0, (Hk, G)))
                out[b, :, i0:i1] = gq.flatten(0, 1)
                dk[b, :, j0:j1] += gk[:, 0]
                dv[b, :, j0:j1] += gv[:, 0]
            else:
                out[b, :, i0:i1] = o.flatten(0, 1)
                lse[b, :, i0:i1] = torch.where(total == 0, -math.inf, top + total.log())[..., 0].flatten(0, 1)
    return (out, dk, dv) if back else (out, lse)
