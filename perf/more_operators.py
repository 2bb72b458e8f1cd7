"""Answering from caches that take fewer bytes, as cases that can be timed and compared: a cache in 8 bits (written, read
back), softmax attention that reads it, and softmax attention of a batch whose sequences share a prefix.

`listed()` names the cases that are quoted, `draw(rng)` gives another one of the same ranges, `prepare(case, seed)` makes
what a program holds before the call, `run(state)` is one pass, `work(case)` what the pass cannot do without and
`exact(case, seed)` the outputs in 64 bits.  `own` chooses between the library's calls and elementary torch operations.

A row (the d features of a token and head) is held as codes c and one fp32 scale s, and stands for c s.  With a = max |row|:
  e4m3  s = 2^ceil(log2(a / 448)), c the nearest e4m3 number to x / s;   int8  s = a / 127 in fp32, c the nearest integer to x / s
(ties to even, s at least 2^-126).

Fields of a case:
  op      "cache"         B, Hk, d, Lc, L, store, layout, dtype            L new tokens (ragged where B > 1) into caches of Lc, then all of it back
          "cache_attn"    B, Hq, Hk, Lq, Lk, d, W, causal, eps, kind, store, layout, dtype
          "prefix_attn"   the same and Lp: a prefix of Lp tokens in front of each item's own Lk
  store   "e4m3", "int8"; prefix_attn also "same" (keys and values in the queries' type)
  kind    "cached" (the Lq last tokens of ragged caches), "masked" (inactive tokens too)
  layout  of the new tokens or queries: "bhld" (contiguous heads), "blhd" (as a projection leaves them)
"""
import math

import torch

own = False
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
SMALLEST = 2.0 ** -126   # of a scale


def _cache(name, B, Hk, d, Lc, L, store, layout, dtype):
    return {"name": name, "op": "cache", "B": B, "Hk": Hk, "d": d, "Lc": Lc, "L": L, "store": store, "layout": layout, "dtype": dtype}


def _attn(name, B, Hq, Hk, Lq, Lk, d, W, causal, eps, kind, store, layout, dtype):
    return {"name": name, "op": "cache_attn", "B": B, "Hq": Hq, "Hk": Hk, "Lq": Lq, "Lk": Lk, "d": d, "W": W, "causal": causal,
            "eps": eps, "kind": kind, "store": store, "layout": layout, "dtype": dtype}


def _prefix(name, Lp, *rest):
    return {**_attn(name, *rest), "op": "prefix_attn", "Lp": Lp}


ALL = 1 << 20   # a band that reaches everything


def listed():
    return [
        # the newest token of 8 sequences, and the window of twice the band that the banded attention then takes: launches and latency
        _cache("cache_token", 8, 2, 64, 512, 1, "e4m3", "blhd", "bf16"),
        # the longest context, from the projections' layout into the cache and back
        _cache("cache_prompt", 1, 2, 64, 262144, 262144, "e4m3", "blhd", "bf16"),
        # a later piece of ragged prompts in fp32, sizes that fit nothing
        _cache("cache_ragged", 3, 4, 128, 20011, 5003, "int8", "bhld", "f32"),
        # answering: one token of each of 4 sequences against ragged caches
        _attn("answer_token", 4, 8, 2, 1, 65536, 64, ALL, True, 1.0, "cached", "e4m3", "bhld", "bf16"),
        # the same with more and wider heads
        _attn("answer_wide", 8, 16, 4, 1, 32768, 128, ALL, True, 1.0, "cached", "int8", "blhd", "bf16"),
        # a few fp32 queries on a short, padded cache with inactive tokens, narrow band, rows that are left empty
        _attn("answer_masked", 2, 4, 4, 5, 701, 32, 64, False, 1.0, "masked", "e4m3", "bhld", "f32"),
        # the next piece of a long prompt against all that is in the cache
        _attn("answer_chunk", 1, 8, 2, 2048, 16384, 64, ALL, True, 1.0, "cached", "e4m3", "blhd", "bf16"),
        # a few samples of one short prompt in fp32, odd sizes, a band that ends inside the prefix
        _prefix("prefix_odd", 1003, 3, 6, 2, 3, 77, 32, 300, True, 0.5, "masked", "same", "bhld", "f32"),
        # one token of each of 32 answers to one long prompt
        _prefix("prefix_token", 65536, 32, 8, 2, 1, 1024, 64, ALL, True, 1.0, "cached", "same", "blhd", "bf16"),
        # the same on 8-bit caches, wide heads, more answers, longer ones
        _prefix("prefix_token8", 16384, 64, 16, 4, 1, 2048, 128, ALL, True, 1.0, "cached", "int8", "bhld", "bf16"),
        # five drafted tokens of each of 16 answers on the longest context
        _prefix("prefix_draft", 262144, 16, 8, 2, 5, 512, 64, ALL, True, 1.0, "cached", "e4m3", "blhd", "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _pairs(c):
    """Expected pairs of a query and a key for one query head of the whole batch: with an item's own keys, with the prefix."""
    masked = c["kind"] == "masked"
    p = torch.arange(c["Lq"], dtype=torch.float64) + max(0.75 * c["Lk"] - c["Lq"], 0)
    hi = torch.clamp(p if c["causal"] else p + c["W"], max=0.75 * c["Lk"] - 1)
    mine = float(torch.clamp(hi - torch.clamp(p - c["W"], min=0) + 1, min=0).sum()) * c["B"]
    front = float(torch.clamp(c["W"] - p, min=0, max=c.get("Lp", 0)).sum()) * c["B"]
    return (0.8 * mine if masked else mine), (0.8 * front if masked else front)


def work(case):
    c = case
    e, d, B, Hk = (4 if c["dtype"] == "f32" else 2), c["d"], c["B"], c["Hk"]
    row = d + 4 if c["store"] != "same" else d * e   # a key or a value in the cache, its scale with it
    if c["op"] == "cache":
        share = 0.75 if B > 1 and c["L"] > 1 else 1.0
        new, held = share * B * Hk * c["L"], B * Hk * ((c["Lc"] - c["L"]) * (0.75 if B > 1 else 1.0) + share * c["L"])
        return {"bytes": 2 * (new * (d * e + row) + held * row + B * Hk * c["Lc"] * d * e), "flops": 4 * (new + held) * d}
    q = B * c["Hq"] * c["Lq"]
    mine, front = _pairs(c)
    keys = min(0.75 * c["Lk"], c["Lq"] + (1 if c["causal"] else 2) * c["W"]) * B + min(c.get("Lp", 0), c["W"])
    return {"bytes": 2 * q * d * e + 4 * q + 2 * Hk * keys * row, "flops": 4 * d * c["Hq"] * (mine + front)}


def _draw(rng):
    op = rng.choice(["cache", "cache_attn", "cache_attn", "prefix_attn", "prefix_attn"])
    Hk, d, dtype = rng.choice([1, 2, 4]), rng.choice([32, 64, 64, 128]), rng.choice(["f32", "bf16", "bf16"])
    layout, store = rng.choice(["bhld", "blhd"]), rng.choice(["e4m3", "int8"])
    if op == "cache":
        Lc = _log(rng, 16, 262144)
        return _cache("", rng.choice([1, 1, 2, 3, 5, 8]), Hk, d, Lc, min(Lc, rng.choice([1, _log(rng, 1, 64), _log(rng, 1, Lc), Lc])), store, layout, dtype)
    Hq, eps, causal = Hk * rng.choice([1, 2, 3, 4, 8]), rng.choice([0.5, 1.0]), rng.random() < 0.8
    kind = rng.choice(["cached", "cached", "masked"])
    if op == "cache_attn":
        Lk = _log(rng, 16, 131072)
        Lq = min(Lk, rng.choice([1, 1, 1, rng.randint(2, 17), _log(rng, 16, 4096)]))
        return _attn("", rng.choice([1, 2, 3, 4, 8, 16]), Hq, Hk, Lq, Lk, d, rng.choice([ALL, ALL, _log(rng, 4, 4096)]), causal, eps, kind, store, layout, dtype)
    Lk = _log(rng, 4, 4096)
    Lq = min(Lk, rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 8, 128)]))
    return _prefix("", _log(rng, 30, 262144), rng.choice([1, 2, 5, 16, 32, 64, _log(rng, 2, 128)]), Hq, Hk, Lq, Lk, d,
                   rng.choice([ALL, ALL, ALL, _log(rng, 64, 16384)]), causal, eps, kind, rng.choice(["same", store]), layout, dtype)


def _cost(c):
    """Seconds at round rates of the bytes and of the products, the latter weighted by the type."""
    w = work(c)
    return max(w["bytes"] / 5e12, w["flops"] / (1e15 if c["dtype"] == "bf16" else 1e14))


def _scores(c):
    """Scores that the plain form holds at a time."""
    return 0 if c["op"] == "cache" else c["B"] * c["Hq"] * c["Lq"] * (c["Lk"] + c.get("Lp", 0))


def _held(c):
    """Keys that the plain form has in fp32 at a time, in features."""
    return c["d"] * c["Hk"] * (c["B"] * c.get("Lc", c.get("Lk", 0)) + c.get("Lp", 0))


def draw(rng):
    """A case of the ranges above that costs no more than the largest listed one, of plain and of library operations."""
    cases = listed()
    most = [max(f(c) for c in cases) for f in (_cost, _scores, _held)]
    while True:
        c = _draw(rng)
        if all(f(c) <= m for f, m in zip((_cost, _scores, _held), most)):
            del c["name"]
            return c


# ------------------------------------------------------------------------------------------------ inputs
def _heads(g, B, H, L, c):
    """Activations as a projection makes them: some features larger throughout, some tokens larger than others."""
    d = c["d"]
    big = 1 + 3 * (torch.rand((H, 1, d), generator=g, device="cuda") > 0.95).float()
    x = torch.randn((B, H, L, d), generator=g, device="cuda") * big * torch.exp(0.3 * torch.randn((B, H, L, 1), generator=g, device="cuda"))
    return x


def _laid(x, c):
    x = x.to(DTYPES[c["dtype"]])
    return x.transpose(1, 2).contiguous().transpose(1, 2) if c["layout"] == "blhd" else x


def _quantise(x, store):
    """Codes and scales of rows (fp32 or narrower), by the definition; borders in 64 bits."""
    a = x.float().abs().amax(-1, keepdim=True)
    if store == "int8":
        s = (a / 127).clamp(min=SMALLEST)
        return (x.double() / s.double()).round().clamp(-127, 127).to(torch.int8), s[..., 0]
    m, e = torch.frexp(a)      # a = m 2^e, 448 = 0.875 2^9
    s = torch.ldexp(torch.ones_like(a), e - 9 + (m > 0.875).int()).clamp(min=SMALLEST)
    return (x.float() / s).to(torch.float8_e4m3fn), s[..., 0]


def _stored(x, c, store):
    """What a program keeps of keys or values: a tensor, or codes and scales."""
    if store == "same":
        return (x.to(DTYPES[c["dtype"]]),)
    return _quantise(x.to(DTYPES[c["dtype"]]), store)


def _pair(k, v):
    return k + v if len(k) == 1 else (k[0], v[0], k[1], v[1])


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    ints = lambda lo, hi, n: torch.randint(lo, hi + 1, (n,), generator=g, device="cuda", dtype=torch.int32)   # noqa: E731
    s, B, Hk = {"case": c}, c["B"], c["Hk"]
    if c["op"] == "cache":
        L, Lc = c["L"], c["Lc"]
        s["k"], s["v"] = _laid(_heads(g, B, Hk, L, c), c), _laid(_heads(g, B, Hk, L, c), c)
        s["cache"] = _pair(*(_stored(_heads(g, B, Hk, Lc, c), c, c["store"]) for _ in range(2)))
        s["start"] = s["new"] = None
        if B > 1:   # ragged: so many are there, so many come
            s["start"], s["new"] = ints((Lc - L + 1) // 2, Lc - L, B), ints((L + 1) // 2, L, B)
        s["len"] = None if B == 1 else s["start"] + s["new"]
        if B == 1 and L < Lc:
            s["start"], s["len"] = torch.full((1,), Lc - L, device="cuda", dtype=torch.int32), None
        return s
    Lq, Lk = c["Lq"], c["Lk"]
    s["q"] = _laid(_heads(g, B, c["Hq"], Lq, c), c)
    s["own"] = _pair(*(_stored(_heads(g, B, Hk, Lk, c), c, c["store"]) for _ in range(2)))
    if c["op"] == "prefix_attn":
        s["prefix"] = _pair(*(_stored(_heads(g, 1, Hk, c["Lp"], c)[0], c, c["store"]) for _ in range(2)))
    s["len_k"] = torch.clamp(ints((Lk + 1) // 2, Lk, B), min=Lq)
    s["start"] = s["len_k"] - Lq
    s["mask_q"] = s["mask_k"] = s["mask_p"] = None
    if c["kind"] == "masked":
        # runs of inactive tokens, some longer than a narrow band
        runs = lambda r, n: (torch.rand((r, (n + 15) // 16), generator=g, device="cuda") > 0.2).repeat_interleave(16, 1)[:, :n].to(torch.uint8).contiguous()   # noqa: E731
        s["mask_k"] = runs(B, Lk)
        s["mask_q"] = (torch.rand((B, Lq), generator=g, device="cuda") > 0.2).to(torch.uint8)
        s["mask_p"] = runs(1, c["Lp"])[0] if c["op"] == "prefix_attn" else None
    return s


# ------------------------------------------------------------------------------------------------ plain forms
def _plain_cache(s):
    """New rows put where they belong, then everything that is held as values in the tokens' type, zeros behind the last."""
    c = s["case"]
    B, L, Lc = c["B"], c["L"], c["Lc"]
    at = torch.arange(Lc, device="cuda")[None]
    l = at - (0 if s["start"] is None else s["start"][:, None])                       # [B, Lc]: which new token belongs there
    new = ((l >= 0) & (l < (L if s["new"] is None else s["new"][:, None]))).expand(B, Lc)[:, None, :]
    pick = l.clamp(0, L - 1).expand(B, Lc).long()
    end = torch.full((B,), Lc, device="cuda") if s["len"] is None else s["len"]
    held = (at < end[:, None])[:, None, :, None]
    out = []
    for x, codes, scale in ((s["k"], s["cache"][0], s["cache"][2]), (s["v"], s["cache"][1], s["cache"][3])):
        q, t = _quantise(x, c["store"])
        bits = codes.view(torch.uint8)
        rows = torch.gather(q.view(torch.uint8), 2, pick[:, None, :, None].expand(bits.shape))
        bits.copy_(torch.where(new[..., None], rows, bits))
        scale.copy_(torch.where(new, torch.gather(t, 2, pick[:, None, :].expand(scale.shape)), scale))
        out += [torch.where(held, codes.float() * scale[..., None], 0.0).to(x.dtype), scale]
    return tuple(out)


def _values(kept):
    """Keys and values in fp32 of what is kept."""
    if len(kept) == 2:
        return kept[0].float(), kept[1].float()
    return kept[0].float() * kept[2][..., None], kept[1].float() * kept[3][..., None]


def _plain_attn(s):
    c = s["case"]
    B, Hq, Hk, Lq, Lk, d, W = (c[x] for x in ("B", "Hq", "Hk", "Lq", "Lk", "d", "W"))
    G = Hq // Hk
    k, v = _values(s["own"])
    p = s["start"][:, None] + torch.arange(Lq, device="cuda")                          # positions behind the prefix
    gap = torch.arange(Lk, device="cuda") - p[..., None]                               # [B, Lq, Lk]
    ok = (gap.abs() <= W) & (torch.arange(Lk, device="cuda") < s["len_k"][:, None, None])
    if c["causal"]:
        ok = ok & (gap <= 0)
    if s["mask_k"] is not None:
        ok = ok & s["mask_k"].bool()[:, None]
    q = s["q"].float().reshape(B, Hk, G * Lq, d) * (1.0 / (c["eps"] * math.sqrt(d)))   # rows g Lq + i
    score = torch.matmul(q, k.transpose(-1, -2).contiguous())
    if c["op"] == "prefix_attn":
        Lp = c["Lp"]
        pk, pv = _values(s["prefix"])
        rows = q.transpose(0, 1).reshape(Hk, B * G * Lq, d)                            # of all items that share a key head
        front = torch.matmul(rows, pk.transpose(-1, -2).contiguous()).view(Hk, B, G * Lq, Lp).transpose(0, 1)
        near = (p[..., None] + Lp - torch.arange(Lp, device="cuda")) <= W
        if s["mask_p"] is not None:
            near = near & s["mask_p"].bool()
        score, ok = torch.cat([front, score], -1), torch.cat([near, ok], -1)
    if s["mask_q"] is not None:
        ok = ok & s["mask_q"].bool()[..., None]
    score = score.view(B, Hk, G, Lq, -1).masked_fill(~ok[:, None, None], -math.inf).view(score.shape)
    top = score.amax(-1, keepdim=True)
    e = torch.exp(score - top.clamp(min=-3e38))
    total = e.sum(-1, keepdim=True)
    if c["op"] == "prefix_attn":
        head = e[..., :c["Lp"]].transpose(0, 1).reshape(Hk, B * G * Lq, c["Lp"])
        o = torch.matmul(e[..., c["Lp"]:].contiguous(), v) + torch.matmul(head, pv).view(Hk, B, G * Lq, d).transpose(0, 1)
    else:
        o = torch.matmul(e, v)
    o = o / torch.where(total > 0, total, 1.0)
    return o.view(B, Hq, Lq, d).to(s["q"].dtype), (top + total.log()).view(B, Hq, Lq)


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    s = state
    c = s["case"]
    if own:
        import paper_2605_08123_amd as ska
        if c["op"] == "cache":
            ska.ska_cache_write(s["cache"], s["k"], s["v"], start=s["start"], len_new=s["new"])
            k, v = ska.ska_cache_read(s["cache"], len_k=s["len"], dtype=s["k"].dtype)
            return k, s["cache"][2], v, s["cache"][3]
        if c["op"] == "cache_attn":
            return ska.ska_cache_attn_fwd(s["q"], s["own"], c["W"], causal=c["causal"], eps=c["eps"], start_q=s["start"], len_k=s["len_k"],
                                          mask_q=s["mask_q"], mask_k=s["mask_k"])
        return ska.ska_prefix_attn_fwd(s["q"], s["prefix"], s["own"], c["W"], causal=c["causal"], eps=c["eps"], start_q=s["start"],
                                       len_k=s["len_k"], mask_q=s["mask_q"], mask_k=s["mask_k"], mask_p=s["mask_p"])
    return _plain_cache(s) if c["op"] == "cache" else _plain_attn(s)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _e4m3_numbers():
    """The 127 numbers from 0 to 448, by exponent and mantissa."""
    return torch.tensor([m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127], dtype=torch.float64, device="cuda")


def _exact_row_values(x, store):
    """(values that the codes of x's rows stand for, scales), searched among all codes."""
    f = x.double()
    a = f.abs().amax(-1, keepdim=True)
    if store == "int8":
        s = torch.clamp((a / 127).float().double(), min=SMALLEST)
        low = torch.floor(f / s)
        rest = f - low * s            # exact: both have 32 bits at most
        up = (2 * rest > s) | ((2 * rest == s) & (low % 2 != 0))
        return torch.clamp(low + up, -127, 127) * s, s[..., 0]
    s = torch.ones_like(a)
    for _ in range(300):              # by doubling and halving: the least power of two that 448 times it reaches the largest
        s = torch.where((448 * s < a), 2 * s, torch.where((448 * s / 2 >= a) & (s > SMALLEST), s / 2, s))
    numbers = _e4m3_numbers()
    between = (numbers[1:] + numbers[:-1]) / 2
    y = f.abs() / s
    i = torch.searchsorted(between, y.contiguous())
    i = i + ((y == between[i.clamp(max=125)]) & (i % 2 == 1))
    return numbers[i.clamp(max=126)] * torch.sign(f) * s, s[..., 0]


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["op"] == "cache":
        out = []
        for x, codes, scale in ((s["k"], s["cache"][0], s["cache"][2]), (s["v"], s["cache"][1], s["cache"][3])):
            value, t = codes.double() * scale.double()[..., None], scale.double()
            rows, new = _exact_row_values(x, c["store"])
            for b in range(c["B"]):
                i = 0 if s["start"] is None else int(s["start"][b])
                n = c["L"] if s["new"] is None else int(s["new"][b])
                value[b, :, i:i + n], t[b, :, i:i + n] = rows[b, :, :n], new[b, :, :n]
                if s["len"] is not None:
                    value[b, :, int(s["len"][b]):] = 0
            out += [value, t]
        return tuple(out)
    return _exact_attn(s)


def _exact_attn(s):
    """By the definition, item by item, a piece of the query rows after another."""
    c = s["case"]
    B, Hq, Hk, Lq, W = (c[x] for x in ("B", "Hq", "Hk", "Lq", "W"))
    P = c.get("Lp", 0)
    out = torch.zeros((B, Hq, Lq, c["d"]), device="cuda", dtype=torch.float64)
    lse = torch.full((B, Hq, Lq), -math.inf, device="cuda", dtype=torch.float64)

    def kept(t, b=None):
        pick = (lambda x: x) if b is None else (lambda x: x[b])
        return [pick(t[i]).double() * (pick(t[i + 2]).double()[..., None] if len(t) == 4 else 1) for i in (0, 1)]

    for b in range(B):
        n = int(s["len_k"][b])
        k, v = (x[:, :n] for x in kept(s["own"], b))
        j = torch.arange(P + n, device="cuda")
        live = torch.ones(P + n, dtype=torch.bool, device="cuda")
        if s["mask_k"] is not None:
            live[P:] = s["mask_k"][b, :n] != 0
        if P:
            pk, pv = kept(s["prefix"])
            k, v = torch.cat([pk, k], 1), torch.cat([pv, v], 1)
            if s["mask_p"] is not None:
                live[:P] = s["mask_p"] != 0
        for i0 in range(0, Lq, 512):
            i1 = min(Lq, i0 + 512)
            p = P + int(s["start"][b]) + torch.arange(i0, i1, device="cuda")[:, None]
            off = (j > p + W) | (j < p - W) | ~live
            if c["causal"]:
                off = off | (j > p)
            if s["mask_q"] is not None:
                off = off | (s["mask_q"][b, i0:i1, None] == 0)
            for h in range(Hk):
                heads = slice(h * (Hq // Hk), (h + 1) * (Hq // Hk))
                a = (s["q"][b, heads, i0:i1].double() @ k[h].transpose(-1, -2)) / (c["eps"] * c["d"] ** 0.5)
                a = torch.where(off, -1e300, a)
                top = a.amax(-1, keepdim=True)
                e = torch.where(off, 0.0, torch.exp(a - top))
                total = e.sum(-1, keepdim=True)
                out[b, heads, i0:i1] = (e @ v[h]) / torch.where(total == 0, 1.0, total)
                lse[b, heads, i0:i1] = torch.where(total == 0, -math.inf, top + total.log())[..., 0]
    return out, lse
