"""Performance cases of the operators behind a model's last layer: the output head as a product of 8-bit
integers, and what is read off its logits (log probabilities, entropy, confidence, top alternatives).

One pass is one call as a serving program makes it: hidden states to logits, or logits to log
probabilities.  Weights, scales and workspaces are what such a program keeps on the device; activations
have the outlier channels of trained models, logits are a background with one dominant entry on most
rows (the share of confident tokens of the package's synthetic workloads).
"""
from __future__ import annotations

import math

import torch

own = False                            # True: the framework's kernels; False: plain torch operations

_FLOAT = {"bf16": torch.bfloat16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp32": 4}


def listed():
    return [
        # One sequence generating: the head of a small vocabulary, weights streamed once for one token.
        _linear("head_t1", 1, 32000, 2048, "bf16", "fp32"),
        # A projection of a small decode batch: a few microseconds, launches and latency.
        _linear("proj_t8", 8, 2048, 2048, "bf16", "bf16"),
        # The ordinary decode batch of a server in front of a large vocabulary.
        _linear("head_t64", 64, 131072, 4096, "bf16", "fp32"),
        # A ragged prompt with odd sizes in every direction, and a bias per output.
        _linear("head_ragged_t333", 333, 50257, 1971, "bf16", "bf16", bias=True),
        # An fp32 model's projection from the wide side, a mixed batch of prompt chunks.
        _linear("proj_fp32_t700", 700, 2048, 5632, "fp32", "fp32"),
        # Up-projection of a long prompt whose tokens were quantised once for several products.
        _linear("codes_t4096", 4096, 14336, 4096, "codes", "bf16"),
        # Logits of every position of a long prompt (prompt scoring): the largest product.
        _linear("head_prompt_t4096", 4096, 131072, 4096, "bf16", "bf16"),
        # Confidence and next token of one sequence: latency only.
        _logprobs("logp_t1", 1, 32000, "fp32", given=1, top=1),
        # A decode batch whose clients asked for the longest list of alternatives.
        _logprobs("logp_t64", 64, 131072, "fp32", given=1, top=20),
        # Four answers scored at every position of ragged prompts, rows of an odd length.
        _logprobs("logp_ragged_t1999", 1999, 50257, "bf16", given=4, top=5),
        # Decoding under a grammar: most of a row is masked, on some rows all but a few dozen tokens.
        _logprobs("logp_masked_t128", 128, 151001, "fp32", given=1, top=10, masked=0.75, pad=7),
        # Log probabilities of a long prompt, with a few alternatives each.
        _logprobs("logp_prompt_t4096", 4096, 131072, "bf16", given=1, top=8),
    ]


def _linear(name, tokens, outputs, inner, x, out, bias=False):
    """x: "bf16" / "fp32" (quantised in the call) or "codes" (8-bit codes and scales given)."""
    return {"name": name, "kind": "linear", "tokens": tokens, "outputs": outputs, "inner": inner, "x": x, "out": out, "bias": bias}


def _logprobs(name, tokens, vocab, dtype, given, top, masked=0.0, pad=0):
    """masked: share of the rows with masked entries; pad: elements between one row's end and the next."""
    return {"name": name, "kind": "logprobs", "tokens": tokens, "vocab": vocab, "dtype": dtype, "given": given, "top": top,
            "masked": masked, "pad": pad}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.55:
        x = rng.choice(["bf16", "bf16", "fp32", "codes"])
        c = _linear("", _log_int(rng, 1, 4096), _log_int(rng, 500, 131072), _log_int(rng, 64, 8192), x, rng.choice(["bf16", "fp32"]),
                    bias=rng.random() < 0.3)
        if rng.random() < 0.5:                               # most models' sizes are round, most batches are not
            c["inner"] = max(64, c["inner"] // 64 * 64)
            c["outputs"] = max(512, c["outputs"] // 128 * 128)
        biggest = next(w for w in map(work, listed()) if w["flops"] == max(work(k)["flops"] for k in listed()))
        while work(c)["flops"] > biggest["flops"] or work(c)["bytes"] > biggest["bytes"]:
            c["tokens"] = max(1, c["tokens"] // 2)
            c["outputs"] = max(500, c["outputs"] - c["outputs"] // 4)
    else:
        c = _logprobs("", _log_int(rng, 1, 4096), _log_int(rng, 1000, 160000), rng.choice(["bf16", "fp32"]), rng.choice([0, 1, 1, 2, 4, 7]),
                      rng.choice([0, 1, 1, 3, 5, 8, 20]), masked=rng.choice([0.0, 0.0, 0.25, 1.0]), pad=rng.choice([0, 0, 0, 8, 13]))
        while c["tokens"] * c["vocab"] * _BYTES[c["dtype"]] > 4096 * 131072 * 2:
            c["tokens"] = max(1, c["tokens"] // 2)
    c.pop("name")
    return c


# ------------------------------------------------------------------------------------ inputs
def _inputs(case, seed):
    """Everything random of a case, the same for both forms and for `exact`."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    if case["kind"] == "linear":
        return _linear_inputs(case, g)
    T, V = case["tokens"], case["vocab"]
    z = torch.empty((T, V + case["pad"]), dtype=_FLOAT[case["dtype"]], device="cuda")
    for t in range(0, T, 512):
        z[t:t + 512] = torch.randn((min(512, T - t), V + case["pad"]), generator=g, device="cuda") * 3.0
    logits = z[:, :V]
    rows = torch.arange(T, device="cuda")
    hot = torch.randint(0, V, (T,), generator=g, device="cuda")
    sure = torch.rand((T,), generator=g, device="cuda") < 0.8
    tokens = torch.randint(0, V, (T, case["given"]), generator=g, device="cuda")
    if case["given"]:                                        # the first of the given tokens is mostly the likely one
        likely = torch.rand((T,), generator=g, device="cuda") < 0.6
        tokens[:, 0] = torch.where(likely, hot, tokens[:, 0])
    logits[rows[sure], hot[sure]] += 16.0
    if case["masked"]:
        # what the grammar allows: on half of the masked rows 40 tokens, on the others a tenth of the vocabulary; always the given ones
        m = rows[torch.rand((T,), generator=g, device="cuda") < case["masked"]]
        for t in m.tolist():
            few = t % 2 == 0
            keep = torch.zeros((V,), dtype=torch.bool, device="cuda")
            n = 40 if few else max(40, V // 10)
            keep[torch.randperm(V, generator=g, device="cuda")[:n]] = True
            keep[tokens[t]] = True
            logits[t].masked_fill_(~keep, -math.inf)
    return {"logits": logits, "tokens": tokens.to(torch.int32)}


def _linear_inputs(case, g):
    T, N, K = case["tokens"], case["outputs"], case["inner"]
    ld = (K + 15) // 16 * 16                                 # rows of codes start on 16 bytes, padding is zero
    w = torch.zeros((N, ld), dtype=torch.int8, device="cuda")
    for n in range(0, N, 16384):
        r = torch.randn((min(16384, N - n), K), generator=g, device="cuda")
        w[n:n + 16384, :K] = (r * 34.0).round_().clamp_(-127, 127).to(torch.int8)
    w_scale = (0.02 / 34.0) * (1.0 + 0.2 * torch.rand((N,), generator=g, device="cuda"))
    x = torch.randn((T, K), generator=g, device="cuda")
    outlier = torch.rand((K,), generator=g, device="cuda") < 0.01
    x = x * torch.where(outlier, 12.0, 1.0) * torch.exp(0.3 * torch.randn((T, 1), generator=g, device="cuda"))
    state = {"w": w[:, :K], "w_scale": w_scale,
             "bias": torch.randn((N,), generator=g, device="cuda") * 0.1 if case["bias"] else None}
    if case["x"] == "codes":
        a = x.abs().amax(dim=1, keepdim=True)
        q = torch.zeros((T, ld), dtype=torch.int8, device="cuda")
        q[:, :K] = (x * (127.0 / a)).round_().to(torch.int8)
        state.update(x=q[:, :K], x_scale=(a / 127.0).reshape(T))
    else:
        state.update(x=x.to(_FLOAT[case["x"]]), x_scale=None)
    return state


def prepare(case, seed):
    state = _inputs(case, seed)
    state["case"] = case
    if own:
        from paper_2510_12357_amd import binding as mm
        if case["kind"] == "linear":
            out = torch.empty((case["tokens"], case["outputs"]), dtype=_FLOAT[case["out"]], device="cuda")
            state["linear"] = mm.Int8Linear(state["w"], state["w_scale"], state["bias"])
            state["out"] = out
        else:
            state["buffers"] = mm.LogprobBuffers(case["tokens"], case["given"], case["top"], case["vocab"])
    return state


# ------------------------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if own:
        if case["kind"] == "linear":
            return state["linear"](state["x"], x_scale=state["x_scale"], out=state["out"])
        b = state["buffers"].run(state["logits"], state["tokens"])
        return {"token_logp": b.token_logp, "entropy": b.entropy, "conf": b.conf, "top_idx": b.top_idx, "top_logp": b.top_logp}
    return _plain_linear(state) if case["kind"] == "linear" else _plain_logprobs(state)


def _plain_linear(state):
    x, scale = state["x"], state["x_scale"]
    if scale is None:                                        # 127 x / a is next to a border where it is rounded: 64 bits
        a = x.abs().amax(dim=1, keepdim=True).double()
        q = torch.where(a > 0, 127.0 * x.double() / a, 0.0).round().float()
        scale = (a / 127.0).float().reshape(-1)
    else:
        q = x.float()
    out = (q @ state["w"].float().t()) * scale[:, None] * state["w_scale"][None, :]
    if state["bias"] is not None:
        out = out + state["bias"][None, :]
    return out.to(_FLOAT[state["case"]["out"]])


def _plain_logprobs(state):
    z, tokens, n = state["logits"].float(), state["tokens"].long(), state["case"]["top"]
    T, V = z.shape
    m = z.amax(dim=1, keepdim=True)
    d = z - m
    e = torch.exp(d)
    total = e.sum(dim=1, keepdim=True, dtype=torch.float64)  # a long sum, and log(1 + little) on confident rows
    log_total = torch.log(total)
    spread = torch.where(e > 0, e * d, 0.0).sum(dim=1, keepdim=True, dtype=torch.float64)
    lp = lambda v: ((v - m).double() - log_total).float()    # noqa: E731
    ids = torch.arange(V, device=z.device, dtype=torch.int32)
    top = torch.empty((T, n), dtype=torch.int32, device=z.device)
    taken = torch.zeros_like(z, dtype=torch.bool)
    for j in range(n):                                       # the largest that is left, of equal ones the lowest id
        best = torch.where(taken, -math.inf, z).amax(dim=1, keepdim=True)
        top[:, j] = torch.where((z == best) & ~taken, ids, V).amin(dim=1)
        taken.scatter_(1, top[:, j:j + 1].long(), True)
    return {"token_logp": lp(z.gather(1, tokens)), "entropy": (log_total - spread / total).float().reshape(T),
            "conf": (1.0 / total).float().reshape(T), "top_idx": top, "top_logp": lp(z.gather(1, top.long()))}


# ------------------------------------------------------------------------------------ cost and definition
def work(case):
    if case["kind"] == "linear":
        T, N, K = case["tokens"], case["outputs"], case["inner"]
        x = T * K + 4 * T if case["x"] == "codes" else T * K * _BYTES[case["x"]]
        return {"bytes": x + N * K + 4 * N * (2 if case["bias"] else 1) + T * N * _BYTES[case["out"]], "flops": 2 * T * N * K}
    T, V = case["tokens"], case["vocab"]
    return {"bytes": T * V * _BYTES[case["dtype"]] + T * (8 * case["given"] + 8 * case["top"] + 8),
            "flops": 5 * T * V}                              # difference, exponential, two sums and a product


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "linear":
        x = s["x"].double()
        if s["x_scale"] is None:
            # nearest integer to 127 x / a, ties to even, by the remainder of a whole division
            a = x.abs().max(dim=1, keepdim=True).values
            safe = torch.where(a == 0, 1.0, a)
            low = torch.floor(127.0 * x / safe)
            twice = 2.0 * (127.0 * x - low * safe)
            up = (twice > safe) | ((twice == safe) & (torch.remainder(low, 2.0) == 1.0))
            x = low + up.double()
            scale = a / 127.0
        else:
            scale = s["x_scale"].double()[:, None]
        out = torch.empty((case["tokens"], case["outputs"]), dtype=torch.float64, device="cuda")
        for n in range(0, case["outputs"], 16384):
            w = s["w"][n:n + 16384].double() * s["w_scale"][n:n + 16384, None].double()
            out[:, n:n + 16384] = torch.mm(x, w.t().contiguous()) * scale
        return out if s["bias"] is None else out + s["bias"].double()
    parts = {"token_logp": [], "entropy": [], "conf": [], "top_idx": [], "top_logp": []}
    for t in range(0, case["tokens"], 256):
        z = s["logits"][t:t + 256].double()
        m = z.max(dim=1, keepdim=True).values
        # the terms beside one largest entry are added up alone: log(1 + little) keeps its digits
        rest = torch.exp(z - m)
        rest.scatter_(1, z.argmax(dim=1, keepdim=True), 0.0)
        rest = rest.sum(dim=1, keepdim=True)
        logp = (z - m) - torch.log1p(rest)
        p = torch.exp(logp)
        parts["entropy"].append(-torch.where(p > 0, p * logp, 0.0).sum(dim=1))
        parts["conf"].append(1.0 / (1.0 + rest[:, 0]))
        parts["token_logp"].append(torch.gather(logp, 1, s["tokens"][t:t + 256].long()))
        order = torch.sort(s["logits"][t:t + 256].float(), dim=1, descending=True, stable=True).indices[:, :case["top"]]
        parts["top_idx"].append(order.to(torch.int32))
        parts["top_logp"].append(torch.gather(logp, 1, order))
    return {k: torch.cat(v) for k, v in parts.items()}
