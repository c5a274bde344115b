"""Alg. 1 on a toy language model whose layers look back at their sequence: every attention output of the run against the definition in 64 bits on the keys and
values that its own passes wrote, with sequences that end and begin in the same slots and passes that write a position again."""
import numpy as np
import pytest
import torch

from paper_2510_12357_amd import workloads as wl
from paper_2510_12357_amd.alg1_driver import Alg1Batch, SequencePages, ToyAttention, ToyLMDevice
from attention_util import BF16, E4M3, FP32, assert_near, attended, half_step, turn_error, turned, values

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, cache, B, window, norm", [("fp32", None, 7, 0, False), ("bf16", None, 12, 0, True), ("bf16", E4M3, 5, 6, True)])
def test_every_step_sees_its_own_sequence(dtype, cache, B, window, norm):
    cfg = wl.LayerConfig(name="toy", T=1, H=64, E=8, I=48, k_big=4, k_little=2, shared_I=(32,), dtype=dtype, gate_std=0.3, w_std=0.18)
    lm = wl.make_toy_lm(cfg, V=48, L=2, seed=5, head_std=0.5, norm=norm)
    at = ToyAttention.random(cfg, 2, 6, 2, 32, seed=3, page_size=4, cache_dtype=cache, window=window)
    dev = ToyLMDevice.upload(lm, attention=at)
    rec = []
    run = Alg1Batch(dev, B, wl.make_prompt_tokens(3, 60, 48), max_new=11, record=rec)
    for _ in range(45):
        run.step()
    kv = {}                                                  # (layer, sequence) -> rows by position
    again = longest = 0
    for r in rec:
        pos = [p - 1 for p in r["pos"]]
        for l, a in enumerate(r["attention"]):
            q, k, v = a["rows"].split([6, 2, 2], dim=1)
            p = torch.tensor(pos, dtype=torch.int32)
            assert_near(a["turned"], turned(q, p, at.rotary.freq, "half"), turn_error(q, at.rotary.freq, "half"), q.dtype)
            for b, s in enumerate(r["seq_id"]):
                if s < 0:
                    assert (a["out"][b] == 0).all()
                    continue
                rows = kv.setdefault((l, s), {})
                again += l == 0 and pos[b] in rows           # the big pass writes what the little one wrote
                rows[pos[b]] = (k[b], v[b])
                assert sorted(rows) == list(range(pos[b] + 1))
                n = pos[b] + 1
                lo = max(0, n - window) if window else 0
                longest = max(longest, n)
                ks, vs = (torch.stack([rows[i][j] for i in range(lo, n)]) for j in (0, 1))
                kt, vt = turned(ks, torch.arange(lo, n), at.rotary.freq, "half"), vs.double()
                # stored rows: rounded to the cache's type, 8-bit ones to half a step of their codes; a channel's error goes into scores and values
                own = 0.0 if at.cache_dtype is FP32 else half_step(BF16) if at.cache_dtype is BF16 else 2.0 ** -4 + 2.0 ** -10
                dk = kt.abs() * own + turn_error(ks, at.rotary.freq, "half")
                dv = vt.abs() * own
                if at.cache_dtype is E4M3:                   # the smallest codes are 2^-9 of the row's scale apart
                    dk, dv = (d + t.abs().amax(-1, keepdim=True) / 448 * 2.0 ** -10 for d, t in ((dk, kt), (dv, vt)))
                qd = a["turned"][b].double().view(2, 3, 32)
                want, _, err, _ = attended(a["turned"][b], (kt, vt), 32 ** -0.5)
                ds = torch.einsum("hgd,nhd->hgn", qd.abs(), dk) * 32 ** -0.5
                score = torch.softmax(torch.einsum("hgd,nhd->hgn", qd, kt) * 32 ** -0.5, dim=2)
                # p changes by at most e^(2 ds) - 1 of itself, the sum of values by that and by the values' own error
                more = torch.einsum("hgn,nhd->hgd", score * torch.expm1(2 * ds.amax(dim=2, keepdim=True)), vt.abs() + dv) + torch.einsum("hgn,nhd->hgd", score, dv)
                assert_near(a["out"][b], want, err + more.reshape(6, 32), a["out"].dtype)
    ends = {f[0] for f in run.finished}
    # what the last step rejected is not run again here
    assert again == run.n_fallbacks - int(run.big.sum()) > 0 and len(ends) > B and longest >= 11
    # pages are given back: those in use are what the running sequences need
    need = sum(-(-len(run.tokens[b]) // 4) for b in range(B) if run.seq_id[b] >= 0)
    assert len(run.pages.free) >= run.pages.n_pages - need and sorted(run.pages.free + run.pages.host[run.pages.host >= 0].tolist()) == list(range(run.pages.n_pages))


def test_pages_are_taken_as_sequences_grow():
    p = SequencePages(2, 9, 4, "cuda")
    for pos in range(9):
        p.reach(0, pos)
    p.reach(1, 0)
    assert (p.upload().cpu().numpy() == p.host).all() and (p.host >= 0).sum() == 4 and len(set(p.host[p.host >= 0].tolist())) == 4
    p.give_back(0)
    assert len(p.free) == 5 and (p.upload().cpu().numpy()[0] == -1).all()
    cfg = wl.LayerConfig(name="toy", T=1, H=64, E=8, I=48, k_big=4, k_little=2, dtype="bf16", gate_std=0.3, w_std=0.18)
    with pytest.raises(ValueError, match="per layer"):
        ToyLMDevice.upload(wl.make_toy_lm(cfg, V=32, L=1, seed=1), attention=ToyAttention.random(cfg, 2, 2, 1, 32))
