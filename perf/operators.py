"""Cases, plain forms and exact values of the operators on a key / value cache held in 4 bits: attention over it (`attention`), the
attention weight its entries gather (`weigh`), the quantising append, read back (`append`), and eviction by that weight (`evict`).

The cache holds groups of 32 values along the head dimension as 4-bit floating point codes (sign, magnitude among 0, 0.5, 1, 1.5, 2, 3, 4, 6) with
one power of two per group (a byte, exponent + 127; 255 marks a group that reads as NaN).  Pages, one table for all layers:
codes [layers, pages, KV heads, page size, D / 2], scales [layers, pages, KV heads, page size, D / 32], mass and position [layers, pages, KV heads, page size].
"""
import math
import random

import numpy as np
import torch

own = False

GROUP = 32
LEAST, MOST = -23, 13   # exponents of a group
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ---- the cases ------------------------------------------------------------------------------------------------

def _attention(name, n, t, hq, hkv, d, lo, hi, page, dtype, window, ragged):
    return dict(name=name, op="attention", n=n, t=t, hq=hq, hkv=hkv, d=d, lo=lo, hi=hi, page=page, dtype=dtype, window=window, ragged=ragged)


def _weigh(name, n, t, hq, hkv, d, lo, hi, page, dtype, ragged):
    return dict(name=name, op="weigh", n=n, t=t, hq=hq, hkv=hkv, d=d, lo=lo, hi=hi, page=page, dtype=dtype, window="none", ragged=ragged)


def _append(name, n, t, layers, hkv, d, lo, hi, page, dtype, ragged):
    return dict(name=name, op="append", n=n, t=t, layers=layers, hkv=hkv, d=d, lo=lo, hi=hi, page=page, dtype=dtype, ragged=ragged)


def _evict(name, n, layers, hkv, d, entries, budget, sink, recent, page):
    return dict(name=name, op="evict", n=n, layers=layers, hkv=hkv, d=d, entries=entries, budget=budget, sink=sink, recent=recent, page=page)


def listed():
    return [
        # one new token of one sequence of the 1.7 B shape behind 512: latency
        _attention("attention, one token", 1, 1, 16, 8, 128, 512, 512, 16, "bf16", "causal", False),
        # a block of the tiny fp32 model; an odd cache length
        _attention("attention, fp32 block", 2, 4, 4, 2, 64, 77, 129, 16, "fp32", "block", False),
        # draft of the 4 B shape: eight sequences of 1024 to 4096, a block of 8 that is partly committed
        _attention("attention, ragged draft", 8, 8, 32, 8, 128, 1024, 4096, 16, "bf16", "block", True),
        # single tokens of 32 sequences of the MoE shape at every length up to 2048, empty caches among them
        _attention("attention, ragged tokens", 32, 1, 16, 4, 128, 0, 2048, 16, "bf16", "causal", False),
        # single tokens behind long caches: the cache's bytes are all there is
        _attention("attention, long tokens", 4, 1, 32, 8, 128, 60000, 65536, 64, "bf16", "causal", False),
        # verification of the 8 B shape: windows of 2 x 16 rows behind 8192
        _attention("attention, verification", 16, 32, 32, 8, 128, 8192, 8192, 16, "bf16", "verify", False),
        # the weights of one token's row, odd lengths and pages
        _weigh("weigh, one token", 3, 1, 16, 8, 64, 500, 777, 24, "fp32", False),
        # the weights of a verification of the 8 B shape
        _weigh("weigh, verification", 16, 32, 32, 8, 128, 8192, 8192, 16, "bf16", False),
        # the accepted prefixes of a step of the 8 B shape, all 36 layers
        _append("append, a step", 16, 16, 36, 8, 128, 100, 300, 16, "bf16", True),
        # a chunk of a prompt, fp32 rows, odd pages
        _append("append, prompt chunk", 4, 192, 8, 8, 128, 0, 200, 24, "fp32", True),
        # a bounded cache of 4096 entries that a few steps have grown past its budget
        _evict("evict, a few", 16, 4, 8, 128, 4160, 4096, 4, 256, 16),
        # a long prompt cut down to an eighth
        _evict("evict, most", 2, 2, 8, 128, 32768, 4096, 16, 512, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attention", "attention", "attention", "weigh", "append", "evict"])
    hkv, d, page = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128, 128, 256]), rng.choice([8, 16, 16, 24, 64, 100])
    if op in ("attention", "weigh"):
        n, t, group = _log(rng, 1, 32), _log(rng, 1, 64), rng.choice([1, 2, 4, 4, 7, 8])
        hi = max(1, min(_log(rng, 1, 65536), (1 << 20) * 128 // (d * n * hkv), (1 << 25) // (n * hkv * t * group)))
        lo = rng.choice([0, hi // 3, hi])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        if op == "weigh":
            return {k: v for k, v in _weigh("", n, t, hkv * group, hkv, d, lo, hi, page, dtype, rng.random() < 0.5).items() if k != "name"}
        window = rng.choice(["causal", "block", "verify", "none"])
        return {k: v for k, v in _attention("", n, t, hkv * group, hkv, d, lo, hi, page, dtype, window, rng.random() < 0.5).items() if k != "name"}
    if op == "append":
        n, t = _log(rng, 1, 32), _log(rng, 1, 192)
        layers = max(1, min(rng.randint(1, 36), (1 << 23) // (n * t * hkv * d)))
        hi = _log(rng, 1, 1000)
        return {k: v for k, v in _append("", n, t, layers, hkv, d, rng.choice([0, hi // 2, hi]), hi, page, rng.choice(["bf16", "bf16", "fp32"]), rng.random() < 0.7).items() if k != "name"}
    n, entries = _log(rng, 1, 16), _log(rng, 40, 32768)
    layers = max(1, min(rng.randint(1, 8), (1 << 22) // (n * hkv * entries)))
    budget = max(32, rng.choice([entries - rng.randint(1, 8), entries * 7 // 8, entries // 2, entries // 8]))
    return {k: v for k, v in _evict("", n, layers, hkv, d, entries, budget, rng.choice([0, 4, 16]), rng.choice([0, budget // 16, budget // 2]), page).items() if k != "name"}


def _lengths(case):
    """Cache lengths and row counts of the sequences: the case's own, whatever the seed."""
    rng = random.Random(repr(sorted((k, v) for k, v in case.items() if k != "name")))
    if case["op"] == "evict":
        return [case["entries"]] * case["n"], [0] * case["n"]
    lens = [rng.randint(case["lo"], case["hi"]) for _ in range(case["n"])]
    if case["lo"] < case["hi"]:
        lens[rng.randrange(case["n"])] = case["hi"]
    rows = [rng.randint(0 if case["n"] > 1 else 1, case["t"]) if case["ragged"] else case["t"] for _ in range(case["n"])]
    return lens, rows


def _entry_bytes(d):
    return 2 * (d // 2 + d // GROUP)


def work(case):
    lens, rows = _lengths(case)
    d, hkv = case["d"], case["hkv"]
    size = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "attention":
        cached = sum(s for s, r in zip(lens, rows) if r)
        total = sum(rows)
        inner = 0 if case["window"] == "none" else sum(r * r if case["window"] == "block" else r * (r + 1) // 2 for r in rows)
        read = cached * hkv * _entry_bytes(d) + total * case["hq"] * (2 * d * size + 4) + (0 if case["window"] == "none" else 2 * total * hkv * d * size)
        return {"bytes": read, "flops": 4 * d * case["hq"] * (sum(s * r for s, r in zip(lens, rows)) + inner)}
    if case["op"] == "weigh":
        cached = sum(s for s, r in zip(lens, rows) if r)
        return {"bytes": cached * hkv * (_entry_bytes(d) // 2 + 8) + sum(rows) * case["hq"] * (d * size + 4),
                "flops": 2 * d * case["hq"] * sum(s * r for s, r in zip(lens, rows))}
    if case["op"] == "append":   # rows in, codes out, codes in, values out
        per = case["layers"] * sum(rows) * hkv
        return {"bytes": per * (2 * _entry_bytes(d) + 8 + 4 * d * size), "flops": 0}
    lists, e, b = case["n"] * case["layers"] * hkv, case["entries"], case["budget"]
    moves = b * (e - b) / e   # expected: what is kept behind the budget, with weights that do not depend on the slot
    return {"bytes": lists * (8 * e + 2 * moves * (_entry_bytes(d) + 8) if e > b else 0) + 4, "flops": 0}


# ---- what a program has in hand -----------------------------------------------------------------------------------

def _power(e):
    """2 ** e of whole numbers, -126 <= e <= 127, exact."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x):
    """Codes (two a byte, the lower index in the low half) and scale bytes of the groups along the last dimension."""
    g = x.float().unflatten(-1, (-1, GROUP))
    most = g.abs().amax(-1)
    part, exponent = torch.frexp(most)
    e = torch.where(part <= 0.75, exponent - 3, exponent - 2)
    e = torch.where(most > 0, e, LEAST).clamp(LEAST, MOST)
    fine = torch.isfinite(g).all(-1)
    e = torch.where(fine, e, 0)
    y = g * _power(-e).unsqueeze(-1)
    a = y.abs()
    # the nearest level; between two the one of even code
    code = sum(c.to(torch.uint8) for c in (a > 0.25, a >= 0.75, a > 1.25, a >= 1.75, a > 2.5, a >= 3.5, a > 5.0)) + 8 * torch.signbit(y).to(torch.uint8)
    code = torch.where(fine.unsqueeze(-1), code, 0).flatten(-2)
    return (code[..., 0::2] | code[..., 1::2] << 4).contiguous(), torch.where(fine, e + 127, 255).to(torch.uint8)


def _values(codes, scales):
    """What codes and scales stand for, in 32 bits."""
    table = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=codes.device)
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2)
    s = torch.where(scales == 255, math.nan, (scales.to(torch.int32) << 23).view(torch.float32))
    return (table[c.int()].unflatten(-1, (-1, GROUP)) * s.unsqueeze(-1)).flatten(-2)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev).manual_seed(seed)
    host = random.Random(seed)
    lens, counts = _lengths(case)
    n, hkv, d, page, layers = case["n"], case["hkv"], case["d"], case["page"], case.get("layers", 1)
    room = case["t"] if case["op"] == "append" else 0
    # pages of the sequences in any order, some that nobody has; the table is padded with -1
    need = [(s + room + page - 1) // page for s in lens]
    n_pages, wide = sum(need) + 3, max(max(need), 1)
    order = list(range(n_pages))
    host.shuffle(order)
    table = np.full((n, wide), -1, np.int32)
    for i, k in enumerate(need):
        table[i, :k] = [order.pop() for _ in range(k)]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    randn = lambda *shape: torch.randn(*shape, generator=gen, device=dev)  # noqa: E731
    shape = (layers, n_pages, hkv, page)
    s = dict(case=case, table=i32(table), entries=i32(lens), seq_len=i32(lens), status=i32([0] * n), lens=lens, counts=counts)
    # keys with a few channels that are ten times the others', values without; places that no sequence holds are noise, NaN marks among it
    strong = torch.where(torch.rand(hkv, d, generator=gen, device=dev) < 0.03, 10.0, 1.0)
    places = layers * n_pages * hkv * page
    for name, by in (("k", strong), ("v", 0.7)):
        # (one place more than the cache has, for what a padded write puts nowhere)
        codes = torch.randint(0, 256, (places + 1, d // 2), generator=gen, device=dev, dtype=torch.uint8)
        scales = torch.randint(100, 256, (places + 1, d // GROUP), generator=gen, device=dev, dtype=torch.uint8)
        s[name + "_codes"], s[name + "_scales"] = codes[:-1].view(*shape, d // 2), scales[:-1].view(*shape, d // GROUP)
        s["all_" + name] = codes, scales
        if case["op"] != "append":
            free = torch.ones(n_pages, page, dtype=torch.bool, device=dev)
            for i in range(n):
                at = torch.arange(lens[i], device=dev)
                free[s["table"][i].long()[at // page], at % page] = False
            for layer in range(layers):
                c, e = _quantise(randn(n_pages, page, hkv, d) * by)
                s[name + "_codes"][layer] = c.transpose(1, 2)
                s[name + "_scales"][layer] = torch.where(free[:, :, None, None], 255, e).transpose(1, 2)
    s["all_mass"] = torch.rand(places + 1, generator=gen, device=dev)
    s["all_position"] = torch.zeros(places + 1, dtype=torch.int32, device=dev)
    s["mass"], s["position"] = s["all_mass"][:-1].view(shape), s["all_position"][:-1].view(shape)
    dtype = DTYPES[case.get("dtype", "bf16")]
    if case["op"] in ("attention", "weigh"):
        total = max(1, sum(counts))
        row0 = np.cumsum([0] + counts[:-1])
        s.update(row0=i32(row0), n_rows=i32(counts), scale=d ** -0.5, q=(1.5 * randn(total, case["hq"], d)).to(dtype), k=None, v=None, low=None, high=None,
                 out=torch.zeros(total, case["hq"], d, dtype=dtype, device=dev), lse=torch.zeros(total, case["hq"], device=dev))
        if case["window"] != "none":
            s["k"], s["v"] = (randn(total, hkv, d) * strong).to(dtype), (0.7 * randn(total, hkv, d)).to(dtype)
            low, high = [], []
            for r0, c in zip(row0, counts):
                drafted = c // 2   # of a verification: drafted rows, then a [MASK] copy of each that sees what is left of it, and itself
                for r in range(c):
                    low.append(r0)
                    high.append(r0 + c if case["window"] == "block" else r0 + r - drafted if case["window"] == "verify" and r >= drafted else r0 + r + 1)
            if case["window"] != "causal":
                s["low"], s["high"] = i32(low or [0]), i32(high or [0])
        if case["op"] == "weigh":
            s["lse"] = _softmax_parts(s)[1]
    elif case["op"] == "append":
        total = max(1, sum(counts))
        s.update(row0=i32(np.cumsum([0] + counts[:-1])), n_rows=i32(counts), first=i32(lens), lens_before=torch.stack((i32(lens), i32(lens))),
                 k=(randn(layers, total, hkv, d) * strong).to(dtype), v=(0.7 * randn(layers, total, hkv, d)).to(dtype))
        s["k_back"], s["v_back"] = (torch.zeros(layers, n, case["t"], hkv, d, dtype=dtype, device=dev) for _ in range(2))
        s["lens_now"] = s["lens_before"].clone()
        s["entries"], s["seq_len"] = s["lens_now"][0], s["lens_now"][1]
    else:
        # weights as attention leaves them: few large, many small, entries that were never looked at
        s["mass"].copy_(torch.where(s["mass"] < 0.2, 0.0, torch.exp(4 * randn(*shape))))
        slot = torch.arange(wide * page, device=dev)[: case["entries"]]
        for i in range(n):
            s["position"][:, s["table"][i].long()[slot // page], :, slot % page] = (slot * 2 + (slot > 3)).to(torch.int32)[:, None, None]
        s["seq_len"] = i32([2 * case["entries"]] * n)
        s["mass_before"], s["position_before"], s["entries_before"] = s["mass"].clone(), s["position"].clone(), s["entries"].clone()
    if own:
        from paper_2603_25702_amd import kv4
        s["cache"] = kv4.Kv4Cache(k_codes=s["k_codes"], v_codes=s["v_codes"], k_scales=s["k_scales"], v_scales=s["v_scales"], page_table=s["table"],
                                  entries=s["entries"], seq_len=s["seq_len"], status=s["status"], mass=s["mass"], position=s["position"])
        if case["op"] in ("attention", "weigh"):
            s["rows"] = kv4.Kv4Rows(q=s["q"], row0=s["row0"], n_rows=s["n_rows"], T=case["t"], out=s["out"], lse=s["lse"], scale=s["scale"], k=s["k"], v=s["v"],
                                    lo=s["low"], hi=s["high"])
            s["scratch"] = torch.empty(kv4.s2d2_kv4_attention_bytes(s["cache"], n, case["t"], case["hq"]), dtype=torch.uint8, device=dev)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------

def _dense(s, codes, scales, layer, entries):
    """The cached entries of every sequence as one tensor [n, longest, KV heads, D], and which of its places hold one."""
    slot = torch.arange(entries, device=codes.device)
    page = s["table"].clamp(min=0).long()[:, slot // s["case"]["page"]]
    at = (page, slice(None), (slot % s["case"]["page"]).expand_as(page))
    return _values(codes[layer][at], scales[layer][at])


def _softmax_parts(s):
    """Weights of the rows, padded to [n, KV heads, T, group, keys], the logarithm of their sums by row, the keys' values, and the padded rows' places."""
    case = s["case"]
    n, t, hq, hkv, d = case["n"], case["t"], case["hq"], case["hkv"], case["d"]
    dev, longest, total = s["q"].device, max(max(s["lens"]), 1), s["q"].shape[0]
    step = torch.arange(t, device=dev)
    there = step < s["n_rows"][:, None]
    row = torch.where(there, s["row0"][:, None] + step, total - 1).long()
    keys = _dense(s, s["k_codes"], s["k_scales"], 0, longest)
    values = _dense(s, s["v_codes"], s["v_scales"], 0, longest) if case["op"] == "attention" else None
    seen = (torch.arange(longest, device=dev) < s["entries"][:, None])[:, None, :].expand(n, t, longest)
    if s["k"] is not None:
        keys = torch.cat((keys, s["k"].float()[row]), 1)
        low = s["row0"][:, None].expand(n, t) if s["low"] is None else s["low"][row]
        high = row + 1 if s["high"] is None else s["high"][row]
        key_row = s["row0"][:, None, None] + step
        inner = ((key_row >= low[:, :, None]) & (key_row < high[:, :, None]) | (key_row == row[:, :, None])) & there[:, None, :]
        if values is not None:
            values = torch.cat((values, s["v"].float()[row]), 1)
        seen = torch.cat((seen, inner), 2)
    q = s["q"].float()[row].view(n, t, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d)
    score = (q @ keys.permute(0, 2, 3, 1).contiguous()).view(n, hkv, t, hq // hkv, -1) * s["scale"]
    score = score.masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top == -math.inf, 0.0, top))
    summed = weight.sum(-1, keepdim=True)
    lse = torch.where(summed > 0, top + torch.log(summed), -math.inf)
    place = torch.where(there, row, total)
    by_row = torch.zeros(total + 1, hq, device=dev)
    by_row[place] = lse[..., 0].permute(0, 2, 1, 3).reshape(n, t, hq)
    if values is not None:
        values = torch.where(seen.any(1)[:, :, None, None], values, 0.0)
    return weight / torch.where(summed > 0, summed, 1.0), by_row[:total], values, place, row, keys, seen


def _plain_attention(s):
    weight, lse, values, place, _, _, _ = _softmax_parts(s)
    n, hkv, t, group, keys = weight.shape
    o = weight.view(n, hkv, t * group, keys) @ values.permute(0, 2, 1, 3).contiguous()
    out = torch.zeros(s["q"].shape[0] + 1, hkv * group, o.shape[-1], device=o.device)
    out[place] = o.view(n, hkv, t, group, -1).permute(0, 2, 1, 3, 4).reshape(n, t, hkv * group, -1)
    return {"out": out[:-1].to(s["q"].dtype), "lse": lse}


def _plain_weigh(s):
    case = s["case"]
    n, t, hq, hkv, d, page = (case[k] for k in ("n", "t", "hq", "hkv", "d", "page"))
    longest, dev = max(max(s["lens"]), 1), s["q"].device
    step = torch.arange(t, device=dev)
    there = step < s["n_rows"][:, None]
    row = torch.where(there, s["row0"][:, None] + step, s["q"].shape[0] - 1).long()
    keys = _dense(s, s["k_codes"], s["k_scales"], 0, longest)
    q = s["q"].float()[row].view(n, t, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(n, hkv, -1, d)
    score = (q @ keys.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    lse = torch.where(there[:, :, None], s["lse"][row], math.inf).view(n, t, hkv, -1).permute(0, 2, 1, 3).reshape(n, hkv, -1, 1)
    weight = torch.exp(score - torch.where(lse == -math.inf, math.inf, lse)).sum(2)
    slot = torch.arange(longest, device=dev)
    held = slot < s["entries"][:, None]
    at = torch.where(held, s["table"].long()[:, slot // page].clamp(min=0) * page + slot % page, s["mass"].shape[1] * page).reshape(-1)
    gained = torch.zeros(s["mass"].shape[1] * page + 1, hkv, device=dev)
    gained[at] = torch.where(held[:, None, :], weight, 0.0).permute(0, 2, 1).reshape(-1, hkv)
    s["mass"][0] += gained[:-1].view(-1, page, hkv).transpose(1, 2)
    return {"mass": s["mass"]}


def _plain_append(s):
    case = s["case"]
    n, t, page = case["n"], case["t"], case["page"]
    s["lens_now"].copy_(s["lens_before"])
    step = torch.arange(t, device=s["k"].device)
    there = step < s["n_rows"][:, None]
    row = torch.where(there, s["row0"][:, None] + step, 0).long()
    entry = (s["entries"][:, None] + step).long()
    at = s["table"].gather(1, (entry // page).clamp(max=s["table"].shape[1] - 1)).clamp(min=0).long()
    layer = torch.arange(case["layers"], device=at.device)[:, None, None, None]
    head = torch.arange(case["hkv"], device=at.device)
    place = ((layer * s["mass"].shape[1] + at[:, :, None]) * case["hkv"] + head) * page + (entry % page)[:, :, None]   # [layers, n, T, KV heads]
    place = torch.where(there[:, :, None], place, s["all_mass"].numel() - 1)
    back = {}
    for name in ("k", "v"):
        codes, scales = (v[:, row] for v in _quantise(s[name]))
        back[name] = torch.where(there[:, :, None, None], _values(codes, scales), 0.0).to(s["k"].dtype)
        s["all_" + name][0][place] = codes
        s["all_" + name][1][place] = scales
    s["all_position"][place] = (s["seq_len"][:, None] + step)[:, :, None].to(torch.int32).expand(place.shape)
    s["all_mass"][place] = 0.0
    s["lens_now"] += s["n_rows"]
    return {"k": back["k"], "v": back["v"], "mass": s["mass"], "position": s["position"], "entries": s["entries"], "seq_len": s["seq_len"]}


def _plain_evict(s):
    case = s["case"]
    page, e, budget = case["page"], case["entries"], case["budget"]
    s["mass"].copy_(s["mass_before"])
    s["position"].copy_(s["position_before"])
    s["entries"].copy_(s["entries_before"])
    held = {k: s[k] for k in ("k_codes", "v_codes", "k_scales", "v_scales", "mass", "position")}
    if e > budget:
        slot = torch.arange(e, device=s["mass"].device)
        at = s["table"].long()[:, slot // page]
        inside = (slot % page).expand_as(at)
        mass = held["mass"][:, at, :, inside].permute(2, 0, 3, 1)          # [layers, n, KV heads, entries]
        position = held["position"][:, at, :, inside].permute(2, 0, 3, 1)
        kept = (position < case["sink"]) | (position >= s["seq_len"][None, :, None, None] - case["recent"])
        rank = torch.where(kept, math.inf, torch.where(torch.isnan(mass), -math.inf, mass)).sort(dim=-1, descending=True, stable=True).indices
        keep = torch.zeros_like(kept).scatter_(-1, rank[..., :budget], True)
        # the i-th dropped slot below the budget takes the i-th kept one behind it; pairs that there are not move a slot onto itself
        most = min(budget, e - budget)
        hole = torch.where(keep[..., :budget], budget + slot[:budget], slot[:budget]).sort(-1).values[..., :most]
        source = torch.where(keep[..., budget:], slot[budget:], e + slot[budget:]).sort(-1).values[..., :most]
        real = hole < budget
        hole, source = torch.where(real, hole, slot[-1]), torch.where(real, source, slot[-1])
        layer = torch.arange(case["layers"], device=at.device)[:, None, None, None]
        head = torch.arange(case["hkv"], device=at.device)[None, None, :, None]
        seq = torch.arange(case["n"], device=at.device)[None, :, None, None]
        to = (layer, at[seq, hole], head, hole % page)
        source = (layer, at[seq, source], head, source % page)
        for v in held.values():
            v[to] = v[source]
        s["entries"].fill_(budget)
    return {**held, "entries": s["entries"]}


def run(s):
    case = s["case"]
    if not own:
        return {"attention": _plain_attention, "weigh": _plain_weigh, "append": _plain_append, "evict": _plain_evict}[case["op"]](s)
    from paper_2603_25702_amd import kv4
    cache = s["cache"]
    if case["op"] == "attention":
        kv4.s2d2_kv4_attention(cache, 0, s["rows"], s["scratch"])
        return {"out": s["out"], "lse": s["lse"]}
    if case["op"] == "weigh":
        kv4.s2d2_kv4_weigh(cache, 0, s["rows"])
        return {"mass": s["mass"]}
    if case["op"] == "append":
        s["lens_now"].copy_(s["lens_before"])
        kv4.s2d2_kv4_append(cache, s["k"], s["v"], s["row0"], s["n_rows"], case["t"])
        kv4.s2d2_kv4_read(cache, s["first"], s["k_back"], s["v_back"])
        return {"k": s["k_back"], "v": s["v_back"], "mass": s["mass"], "position": s["position"], "entries": s["entries"], "seq_len": s["seq_len"]}
    s["mass"].copy_(s["mass_before"])
    s["position"].copy_(s["position_before"])
    s["entries"].copy_(s["entries_before"])
    kv4.s2d2_kv4_evict(cache, case["budget"], 0, case["sink"], case["recent"])
    return {**{k: s[k] for k in ("k_codes", "v_codes", "k_scales", "v_scales", "mass", "position")}, "entries": s["entries"]}


# ---- the definitions, in 64 bits ----------------------------------------------------------------------------------

def _decode(codes, scales):
    """Sign, exponent and fraction of a code, in 64 bits: (-1)^s 2^(x - 1) (1 + f / 2) for x > 0, (-1)^s f / 2 for x = 0."""
    low, high = (codes & 15).double(), (codes >> 4).double()
    c = torch.cat((low[..., None], high[..., None]), -1).reshape(*codes.shape[:-1], -1)
    sign = 1 - 2 * torch.floor(c / 8)
    x, f = torch.floor(c / 2) % 4, c % 2
    magnitude = torch.where(x > 0, torch.exp2(x - 1) * (1 + f / 2), f / 2)
    power = torch.exp2(scales.double() - 127)
    power[scales == 255] = math.nan
    return sign * magnitude * power.repeat_interleave(GROUP, -1)


def _entries_of(s, i, name, count):
    pages = s["table"][i].tolist()
    page = s["case"]["page"]
    codes = [s[name + "_codes"][0, pages[p]] for p in range((count + page - 1) // page)]
    scales = [s[name + "_scales"][0, pages[p]] for p in range((count + page - 1) // page)]
    return _decode(torch.cat(codes, 1)[:, :count], torch.cat(scales, 1)[:, :count])   # [KV heads, entries, D]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("attention", "weigh"):
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        out = torch.zeros(s["q"].shape[0], hq, d, dtype=torch.float64, device="cuda")
        lse = torch.zeros(s["q"].shape[0], hq, dtype=torch.float64, device="cuda")
        mass = s["mass"].double()
        r = 0
        for i, (length, count) in enumerate(zip(s["lens"], s["counts"])):
            rows = range(r, r + count)
            r += count
            if not count:
                continue
            key = _entries_of(s, i, "k", length) if length else torch.zeros(hkv, 0, d, dtype=torch.float64, device="cuda")
            q = s["q"][rows.start:rows.stop].double()
            if case["op"] == "weigh":
                for h in range(hkv if length else 0):
                    mine = slice(h * hq // hkv, (h + 1) * hq // hkv)
                    p = torch.exp(s["scale"] * (q[:, mine].reshape(-1, d) @ key[h].T) - s["lse"][rows.start:rows.stop, mine].double().reshape(-1, 1)).sum(0)
                    at = torch.arange(length, device="cuda")
                    mass[0, s["table"][i].long()[at // case["page"]], h, at % case["page"]] += p
                continue
            value = _entries_of(s, i, "v", length) if length else torch.zeros(hkv, 0, d, dtype=torch.float64, device="cuda")
            seen = torch.ones(count, length, dtype=torch.bool, device="cuda")
            if s["k"] is not None:
                key = torch.cat((key, s["k"][rows.start:rows.stop].double().transpose(0, 1)), 1)
                value = torch.cat((value, s["v"][rows.start:rows.stop].double().transpose(0, 1)), 1)
                inner = torch.eye(count, dtype=torch.bool, device="cuda")
                for a in range(count):
                    lo, hi = (rows.start, rows.start + a + 1) if s["low"] is None else (int(s["low"][rows[a]]), int(s["high"][rows[a]]))
                    inner[a, lo - rows.start:max(hi, lo) - rows.start] = True
                seen = torch.cat((seen, inner), 1)
            for h in range(hq):
                score = s["scale"] * (q[:, h] @ key[h * hkv // hq].T)
                score[~seen] = -math.inf
                lse[rows.start:rows.stop, h] = torch.logsumexp(score, 1)
                out[rows.start:rows.stop, h] = torch.nan_to_num(torch.softmax(score, 1), nan=0.0) @ value[h * hkv // hq]
        return {"mass": mass} if case["op"] == "weigh" else {"out": out, "lse": lse}
    if case["op"] == "append":
        # the nearest value that a group can hold is found among all sixteen; a tie goes to the even code
        level = torch.tensor(LEVELS, dtype=torch.float64, device="cuda")
        favour = torch.tensor([0.0 if c % 2 == 0 else 1e-12 for c in range(8)], dtype=torch.float64, device="cuda")
        back = {}
        for name in ("k", "v"):
            x = s[name].double().unflatten(-1, (-1, GROUP))
            most = x.abs().amax(-1, keepdim=True)
            e = torch.ceil(torch.log2(torch.clamp(most / 6, min=2.0 ** -200))).clamp(LEAST, MOST)
            e = torch.where((6 * torch.exp2(e - 1) >= most) & (e > LEAST), e - 1, e)
            e = torch.where((6 * torch.exp2(e) < most) & (e < MOST), e + 1, e)
            near = torch.zeros_like(x)
            for layer in range(x.shape[0]):
                y = x[layer] / torch.exp2(e[layer])
                near[layer] = level[((y.abs()[..., None] - level).abs() + favour).argmin(-1)] * torch.sign(y)
            value = (near * torch.exp2(e)).flatten(-2)
            held = torch.zeros(case["layers"], case["n"], case["t"], case["hkv"], case["d"], dtype=torch.float64, device="cuda")
            r = 0
            for i, count in enumerate(s["counts"]):
                held[:, i, :count] = value[:, r:r + count]
                r += count
            back[name] = held
        return {**back, "mass": None, "position": None, "entries": None, "seq_len": None}
    # eviction moves entries as they are held (codes and scales bit for bit); list by list, the weights that are left, in the order of the slots
    mass, position = s["mass"].double().cpu().numpy(), s["position"].cpu().numpy()
    table, page, e, budget = s["table"].cpu().numpy(), case["page"], case["entries"], case["budget"]
    if e > budget:
        slot = np.arange(e)
        for i in range(case["n"]):
            at = table[i][slot // page], slot % page
            for layer in range(case["layers"]):
                for h in range(case["hkv"]):
                    m, p = mass[layer, at[0], h, at[1]], position[layer, at[0], h, at[1]]
                    safe = (p < case["sink"]) | (p >= 2 * e - case["recent"])
                    keep = np.zeros(e, bool)
                    keep[np.lexsort((slot, -m, ~safe))[:budget]] = True
                    to, source = slot[:budget][~keep[:budget]], slot[budget:][keep[budget:]]
                    m[to] = m[source]
                    mass[layer, at[0], h, at[1]] = m
    return {"mass": torch.from_numpy(mass), **{k: None for k in ("k_codes", "v_codes", "k_scales", "v_scales", "position", "entries")}}
