"""Performance cases of a decoder's attention step around a paged key-value cache: rotary positions, new keys and
values appended to the cache with the rotation on the way, and the attention of one new token per sequence over it.

One pass is one call as a serving program makes it.  The cache, its page table and the rotation's frequencies are what
such a program keeps on the device; pages of a sequence lie anywhere in the cache, sequences are of different lengths,
an empty slot of the batch has length 0 or position -1.
"""
from __future__ import annotations

import math
import random

import torch

own = False                            # True: the framework's kernels; False: plain torch operations

_FLOAT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": torch.float8_e4m3fn}
_BYTES = {"bf16": 2, "fp32": 4, "e4m3": 1}
_E4M3_MAX = 448.0


def listed():
    return [
        # Queries of one sequence that is generating: latency only.
        _rope("rope_t1", 1, 32, 128, 128, "half", "bf16", far=4096),
        # Queries and keys of a long prompt out of fused projection rows, with frequencies scaled for a longer context.
        _rope("rope_prompt_t4096", 4096, 40, 128, 128, "half", "bf16", far=65536, factor=8.0, fused=8),
        # An fp32 model that turns neighbouring channels of part of an odd-sized head, at far positions.
        _rope("rope_part_t1333", 1333, 7, 80, 48, "interleaved", "fp32", far=1 << 20),
        # One sequence generating: its query, key and value, latency only.
        _append("append_b1", 1, 1, 16, 16, 128, 128, "half", "bf16", "bf16", page=16),
        # The ordinary decode batch: one token of every sequence.
        _append("append_b64", 64, 64, 32, 8, 128, 128, "half", "bf16", "bf16", page=16),
        # Ragged chunks of a few prompts into a cache of 8 bits, an odd number of tokens, padding at the end.
        _append("append_chunk_t2111", 2111, 5, 20, 4, 96, 64, "interleaved", "bf16", "e4m3", page=32),
        # A whole batch of prompts.
        _append("append_prompt_t16384", 16384, 8, 32, 8, 128, 128, "half", "bf16", "bf16", page=64),
        # One short sequence, as many key heads as query heads: latency only.
        _attend("attend_b1_l200", 1, 200, 16, 16, 128, "bf16", "bf16", page=16),
        # The ordinary decode batch of a server: ragged sequences, four query heads to a key head.
        _attend("attend_b64_l8192", 64, 8192, 32, 8, 128, "bf16", "bf16", page=16),
        # One sequence of a very long document.
        _attend("attend_b1_l131072", 1, 131072, 32, 8, 128, "bf16", "bf16", page=64, lse=True),
        # All query heads on one key head, fp32 activations, a sliding window over small pages and capped scores.
        _attend("attend_shared_window", 33, 5000, 71, 1, 64, "fp32", "bf16", page=8, window=1000, softcap=30.0),
        # The largest batch, its cache in 8 bits.
        _attend("attend_b128_l16384_e4m3", 128, 16384, 64, 8, 128, "bf16", "e4m3", page=32),
    ]


def _rope(name, tokens, heads, dim, rotary, layout, dtype, far, factor=1.0, fused=0):
    """fused: further heads (the values) in the rows that the rotated ones are a part of."""
    return {"name": name, "kind": "rope", "tokens": tokens, "heads": heads, "dim": dim, "rotary": rotary, "layout": layout, "dtype": dtype,
            "far": far, "factor": factor, "fused": fused}


def _append(name, tokens, sequences, heads, kv_heads, dim, rotary, layout, dtype, cache, page):
    return {"name": name, "kind": "append", "tokens": tokens, "sequences": sequences, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "rotary": rotary, "layout": layout, "dtype": dtype, "cache": cache, "page": page}


def _attend(name, sequences, longest, heads, kv_heads, dim, dtype, cache, page, window=0, softcap=0.0, lse=False):
    return {"name": name, "kind": "attend", "sequences": sequences, "longest": longest, "heads": heads, "kv_heads": kv_heads, "dim": dim,
            "dtype": dtype, "cache": cache, "page": page, "window": window, "softcap": softcap, "lse": lse}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rope", "append", "attend", "attend"])
    dim = rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256])
    rotary = rng.choice([dim, dim, dim // 2, dim // 4 // 2 * 2])
    layout = rng.choice(["half", "half", "interleaved"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    page = rng.choice([8, 16, 16, 32, 64, 128, 256])
    kv_heads = rng.choice([1, 2, 3, 4, 8, 8, 16])
    if kind == "rope":
        c = _rope("", _log_int(rng, 1, 8192), rng.randint(1, 48), dim, rotary, layout, dtype, _log_int(rng, 100, 1 << 20),
                  factor=rng.choice([1.0, 1.0, 4.0, 32.0]), fused=rng.choice([0, 0, 1, 8]))
    elif kind == "append":
        tokens = _log_int(rng, 1, 16384)
        sequences = tokens if rng.random() < 0.4 and tokens <= 512 else min(tokens, _log_int(rng, 1, 64))
        c = _append("", tokens, sequences, kv_heads * rng.choice([1, 2, 4, 5, 8]), kv_heads, dim, rotary, layout, dtype,
                    rng.choice(["bf16", "bf16", "e4m3", dtype]), page)
    else:
        c = _attend("", _log_int(rng, 1, 256), _log_int(rng, 1, 131072), kv_heads * rng.choice([1, 2, 4, 4, 5, 8, 16, 24]), kv_heads, dim, dtype,
                    rng.choice(["bf16", "bf16", "e4m3", dtype]), page, window=rng.choice([0, 0, 0, 128, 1000, 4096]),
                    softcap=rng.choice([0.0, 0.0, 50.0]), lse=rng.random() < 0.3)
        while c["sequences"] * c["longest"] * kv_heads * dim * c["heads"] // kv_heads > 128 * 16384 * 128 * 64 \
                or c["sequences"] * c["longest"] * kv_heads * dim * _BYTES[c["cache"]] > 128 * 16384 * 128 * 8:
            if c["sequences"] > 1:
                c["sequences"] //= 2
            else:
                c["longest"] //= 2
    big = [work(k) for k in listed() if k["kind"] == kind]
    while work(c)["bytes"] > max(w["bytes"] for w in big) and c.get("tokens", 1) > 1:
        c["tokens"] = c["tokens"] // 2
        if "sequences" in c:
            c["sequences"] = min(c["sequences"], c["tokens"])
    c.pop("name")
    return c


# ------------------------------------------------------------------------------------ inputs
def _lengths(case):
    """Of an attention case: a batch of more than four has an empty slot and a sequence that has just begun."""
    n, longest = case["sequences"], case["longest"]
    rng = random.Random(1000003 * n + longest)
    got = [longest] + [max(1, int(longest * rng.uniform(0.05, 1.0))) for _ in range(n - 1)]
    if n > 4:
        got[1], got[3] = 0, 1
    return got


def _chunks(case):
    """Of an append: (tokens, those before them) of every sequence.  The rest of the tokens is padding."""
    n, T = case["sequences"], case["tokens"]
    rng = random.Random(1000003 * n + T)
    real = T - (T // 50 if n < T else 0)
    if n == T:
        return [(1, rng.randint(0, 2000)) for _ in range(n)]
    cuts = sorted(rng.randint(0, real) for _ in range(n - 1))
    return [(b - a, rng.choice([0, rng.randint(0, 500)])) for a, b in zip([0] + cuts, cuts + [real])]


def _frequencies(case):
    """Radians per position.  With a factor those that turn less than 4 times over the 8192 positions of training are slowed by it, those that
    turn more than once over them partly."""
    r = case["rotary"]
    f = [10000.0 ** (-2.0 * i / r) for i in range(r // 2)]
    factor = case.get("factor", 1.0)
    if factor != 1.0:
        keep = [min(1.0, max(0.0, (8192 * v / (2 * math.pi) - 1.0) / 3.0)) for v in f]
        f = [v * (a + (1.0 - a) / factor) for v, a in zip(f, keep)]
    return f


def _pages(lengths, page, g):
    """A table [sequences, most pages] of shuffled pages (-1 behind a sequence's end), and how many there are."""
    counts = torch.tensor([-(-n // page) for n in lengths], device="cuda")
    total, most = int(counts.sum()), max(1, int(counts.max()))
    n_pages = total + 3
    order = torch.randperm(n_pages, generator=g, device="cuda")[:total]
    table = torch.full((len(lengths), most), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(most, device="cuda")[None, :] < counts[:, None]] = order.to(torch.int32)
    return table, n_pages


def _quantised(x):
    """-> (codes, scales): each row's largest magnitude becomes the largest code."""
    a = x.abs().amax(dim=-1, keepdim=True)
    y = torch.where(a > 0, _E4M3_MAX * x.double() / a.double(), 0.0).float()     # next to a border where it is rounded: 64 bits
    return y.to(torch.float8_e4m3fn), (a / _E4M3_MAX)[..., 0]


def _filled(n_pages, case, g):
    """A cache [pages, key heads, positions, channels] of what earlier steps left: unit values, a few larger channels."""
    heads, page, dim = case["kv_heads"], case["page"], case["dim"]
    gain = 1.0 + 3.0 * (torch.rand((heads, 1, dim), generator=g, device="cuda") < 0.03)
    x = torch.empty((n_pages, heads, page, dim), dtype=_FLOAT[case["cache"]], device="cuda")
    scale = torch.empty((n_pages, heads, page), dtype=torch.float32, device="cuda") if case["cache"] == "e4m3" else None
    step = max(1, (1 << 27) // (heads * page * dim))
    for p in range(0, n_pages, step):
        v = torch.randn((min(step, n_pages - p), heads, page, dim), generator=g, device="cuda") * gain
        if scale is None:
            x[p:p + step] = v.to(x.dtype)
        else:
            a = v.abs().amax(dim=-1, keepdim=True)
            x[p:p + step] = (v * (_E4M3_MAX / a)).to(x.dtype)
            scale[p:p + step] = a[..., 0] / _E4M3_MAX
    return x, scale


def _inputs(case, seed):
    """Everything random of a case, the same for both forms and for `exact`."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = _FLOAT[case["dtype"]]
    if case["kind"] == "attend":
        lengths = _lengths(case)
        table, n_pages = _pages(lengths, case["page"], g)
        k, k_scale = _filled(n_pages, case, g)
        v, v_scale = _filled(n_pages, case, g)
        q = 1.5 * torch.randn((case["sequences"], case["heads"], case["dim"]), generator=g, device="cuda")
        return {"q": q.to(dtype), "k": k, "v": v, "k_scale": k_scale, "v_scale": v_scale, "table": table,
                "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda")}
    T, dim = case["tokens"], case["dim"]
    s = {"freq": torch.tensor(_frequencies(case), dtype=torch.float64, device="cuda"),
         "mscale": 1.0 + 0.1 * math.log(case.get("factor", 1.0))}
    if case["kind"] == "rope":
        rows = torch.randn((T, case["heads"] + case["fused"], dim), generator=g, device="cuda").to(dtype)
        s["x"] = rows[:, :case["heads"]]
        s["pos"] = torch.randint(0, case["far"], (T,), generator=g, device="cuda").to(torch.int32)
        return s
    chunks = _chunks(case)
    s["table"], n_pages = _pages([n + before for n, before in chunks], case["page"], g)
    s["k"], s["k_scale"] = _filled(n_pages, case, g)
    s["v"], s["v_scale"] = _filled(n_pages, case, g)
    h, hk = case["heads"], case["kv_heads"]
    rows = torch.randn((T, h + 2 * hk, dim), generator=g, device="cuda").to(dtype)       # a fused projection
    s["q"], s["new_k"], s["new_v"] = rows[:, :h], rows[:, h:h + hk], rows[:, h + hk:]
    pos, seq = torch.full((T,), -1, dtype=torch.int32), torch.zeros((T,), dtype=torch.int32)
    at = 0
    for i, (n, before) in enumerate(chunks):
        pos[at:at + n] = torch.arange(before, before + n, dtype=torch.int32)
        seq[at:at + n] = i
        at += n
    s["pos"], s["seq"] = pos.to("cuda"), seq.to("cuda")
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = case
    if own:
        from paper_2510_12357_amd import binding as mm
        if case["kind"] != "attend":
            s["rotary"] = mm.Rotary(s["freq"], layout=case["layout"], mscale=s["mscale"])
            x = s["x"] if case["kind"] == "rope" else s["q"]
            s["out"] = torch.empty(x.shape, dtype=x.dtype, device="cuda")
        if case["kind"] != "rope":
            s["cache"] = mm.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if case["kind"] == "attend":
            s["attention"] = mm.DecodeAttention(s["cache"], case["heads"], window=case["window"], softcap=case["softcap"])
            s["out"] = torch.empty_like(s["q"])
            s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda") if case["lse"] else None
    return s


# ------------------------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if case["kind"] == "rope":
        if own:
            return state["rotary"](state["x"], state["pos"], out=state["out"])
        return _turned(state["x"].float(), state["pos"], state).to(state["x"].dtype)
    if case["kind"] == "append":
        if own:
            one_each = case["sequences"] == case["tokens"]
            q = state["cache"].append(state["new_k"], state["new_v"], state["pos"], state["table"], seq=None if one_each else state["seq"],
                                      rotary=state["rotary"], q=state["q"], q_out=state["out"])
        else:
            q = _plain_append(state)
        got = {"q": q, "k": state["k"], "v": state["v"]}
        return got if state["k_scale"] is None else {**got, "k_scale": state["k_scale"], "v_scale": state["v_scale"]}
    if own:
        out = state["attention"](state["q"], state["table"], state["lengths"], case["longest"], out=state["out"], lse=state["lse"])
        return {"out": out, "lse": state["lse"]} if case["lse"] else {"out": out}
    return _plain_attend(state)


def _turned(x, pos, state):
    """Pairs of channels of x [tokens, heads, channels] turned by position times frequency; far positions need their angles in 64 bits."""
    r = 2 * state["freq"].numel()
    angle = pos.double()[:, None] * state["freq"][None, :]
    c, s = ((f(angle) * state["mscale"]).float()[:, None, :] for f in (torch.cos, torch.sin))
    if state["case"]["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], dim=-1).flatten(-2)
    return torch.cat([turned, x[..., r:]], dim=-1)


def _plain_append(state):
    page = state["case"]["page"]
    q = _turned(state["q"].float(), state["pos"], state).to(state["q"].dtype)
    real = state["pos"] >= 0
    pos, seq = state["pos"][real].long(), state["seq"][real].long()
    at, off = state["table"][seq, pos // page].long(), pos % page
    k = _turned(state["new_k"][real].float(), state["pos"][real], state)
    v = state["new_v"][real]
    if state["k_scale"] is None:
        state["k"][at, :, off] = k.to(state["k"].dtype)
        state["v"][at, :, off] = v.to(state["v"].dtype)
        return q
    codes, state["k_scale"][at, :, off] = _quantised(k)
    state["k"].view(torch.uint8)[at, :, off] = codes.view(torch.uint8)
    codes, state["v_scale"][at, :, off] = _quantised(v.float())
    state["v"].view(torch.uint8)[at, :, off] = codes.view(torch.uint8)
    return q


def _read(cache, scale, table):
    """Rows [sequences, key heads, positions, channels] in 32 bits of the pages in the table."""
    p = table.clamp(min=0).long()
    if scale is None:
        x = cache[p].float()
    else:
        x = cache.view(torch.uint8)[p].view(cache.dtype).float() * scale[p][..., None]
    b, n, h, page, dim = x.shape
    return x.transpose(1, 2).reshape(b, h, n * page, dim)


def _plain_attend(state):
    case, q = state["case"], state["q"].float()
    B, H, D = q.shape
    Hk = case["kv_heads"]
    k = _read(state["k"], state["k_scale"], state["table"])
    at = torch.arange(k.shape[2], device="cuda")[None, :]
    n = state["lengths"][:, None]
    seen = at < n
    if case["window"]:
        seen = seen & (at >= n - case["window"])
    s = torch.matmul(k, q.view(B, Hk, H // Hk, D).transpose(2, 3).contiguous()) * (1.0 / math.sqrt(D))
    del k
    if case["softcap"]:
        s = case["softcap"] * torch.tanh(s / case["softcap"])
    s = torch.where(seen[:, None, :, None], s, -math.inf)
    m = s.amax(dim=2, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    e = torch.exp(s - m)
    total = e.sum(dim=2, keepdim=True)
    p = torch.where(total > 0, e / total, 0.0).transpose(2, 3).contiguous()
    out = torch.matmul(p, _read(state["v"], state["v_scale"], state["table"])).view(B, H, D).to(state["q"].dtype)
    return {"out": out, "lse": (m + torch.log(total)).view(B, H)} if case["lse"] else {"out": out}


# ------------------------------------------------------------------------------------ cost and definition
def work(case):
    b = _BYTES[case["dtype"]]
    if case["kind"] == "rope":
        n = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * b + 4 * case["tokens"] + 4 * case["rotary"],
                "flops": 3 * case["tokens"] * case["heads"] * case["rotary"]}
    row = case["dim"] * _BYTES[case["cache"]] + (4 if case["cache"] == "e4m3" else 0)     # of the cache
    if case["kind"] == "append":
        tokens = sum(n for n, _ in _chunks(case))
        q, kv = case["tokens"] * case["heads"] * case["dim"], 2 * tokens * case["kv_heads"]
        return {"bytes": 2 * q * b + kv * (case["dim"] * b + row) + 8 * case["tokens"] + 4 * case["rotary"],
                "flops": 3 * case["rotary"] * (case["tokens"] * case["heads"] + tokens * case["kv_heads"])}
    seen = [min(n, case["window"]) if case["window"] else n for n in _lengths(case)]
    q = case["sequences"] * case["heads"] * case["dim"]
    return {"bytes": 2 * sum(seen) * case["kv_heads"] * row + 2 * q * b + 4 * sum(-(-n // case["page"]) for n in seen) + 4 * case["sequences"],
            "flops": 4 * sum(seen) * case["heads"] * case["dim"]}


def _exact_turn(x, s):
    """The rotation as a product of complex numbers in 64 bits."""
    half, layout = s["freq"].numel(), s["layout"]
    x = x.double()
    out = x.clone()
    angle = s["pos"].double().reshape(-1, 1, 1) * s["freq"]
    w = torch.polar(torch.full_like(angle, s["mscale"]), angle)
    re, im = (slice(0, half), slice(half, 2 * half)) if layout == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
    z = torch.complex(x[..., re].contiguous(), x[..., im].contiguous()) * w
    out[..., re], out[..., im] = z.real, z.imag
    return out


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rope":
        return _exact_turn(s["x"], {**s, "layout": case["layout"]})
    if case["kind"] == "append":
        s["layout"] = case["layout"]
        new = {"k": _exact_turn(s["new_k"], s), "v": s["new_v"].double()}
        got = {"q": _exact_turn(s["q"], s)}
        slot = s["table"].long()[s["seq"].long(), (s["pos"].long() // case["page"]).clamp(min=0)] * case["page"] + s["pos"].long() % case["page"]
        slot = slot[s["pos"] >= 0]
        for name in ("k", "v"):
            pages, heads, page, dim = s[name].shape
            rows = s[name].float().double().permute(0, 2, 1, 3).reshape(pages * page, heads, dim)     # by slot
            value = new[name][s["pos"] >= 0]
            if s[name + "_scale"] is not None:
                # the value that a code stands for, in units of its scale and before it is rounded
                scales = s[name + "_scale"].double().permute(0, 2, 1).reshape(pages * page, heads)
                scale = value.abs().max(dim=2).values / _E4M3_MAX
                scales[slot] = scale
                got[name + "_scale"] = scales.reshape(pages, page, heads).permute(0, 2, 1).contiguous()
                value = value / scale[..., None]
            rows[slot] = value
            got[name] = rows.reshape(pages, page, heads, dim).permute(0, 2, 1, 3).contiguous()
        return got
    B, H, D = s["q"].shape
    Hk = case["kv_heads"]
    out = torch.zeros((B, H, D), dtype=torch.float64, device="cuda")
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(_lengths(case)):
        first = max(0, n - case["window"]) if case["window"] else 0
        if n == 0:
            continue
        at = torch.arange(first, n, device="cuda")
        page, off = s["table"][b].long()[at // case["page"]], at % case["page"]
        for h in range(Hk):
            k, v = s["k"].view(torch.uint8).view(s["k"].shape[:3] + (-1,))[page, h, off], s["v"].view(torch.uint8).view(s["k"].shape[:3] + (-1,))[page, h, off]
            k, v = (x.view(s["k"].dtype).float().double() for x in (k, v))
            if s["k_scale"] is not None:
                k = k * s["k_scale"][page, h, off].double()[:, None]
                v = v * s["v_scale"][page, h, off].double()[:, None]
            group = slice(h * (H // Hk), (h + 1) * (H // Hk))
            z = torch.mm(s["q"][b, group].double(), k.t().contiguous()) / math.sqrt(D)
            if case["softcap"]:
                z = case["softcap"] * torch.tanh(z / case["softcap"])
            lse[b, group] = torch.logsumexp(z, dim=1)
            out[b, group] = torch.mm(torch.softmax(z, dim=1), v)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}
