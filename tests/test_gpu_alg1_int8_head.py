"""Alg. 1 on a toy language model with a vocabulary beyond the router's: the head in 8-bit integers, the confidence and the next token read
off with the log probabilities, checked against the codes in 64 bits and against the loop's own rules."""
import numpy as np
import pytest
import torch

from paper_2510_12357_amd import binding as mm
from paper_2510_12357_amd import workloads as wl
from paper_2510_12357_amd.alg1_driver import Alg1Batch, ToyLMDevice

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, V, B", [("bf16", 3001, 12), ("fp32", 700, 5), ("bf16", 48, 9)])
def test_alg1_with_an_8_bit_head(dtype, V, B):
    cfg = wl.LayerConfig(name="toy", T=1, H=64, E=8, I=48, k_big=4, k_little=2, shared_I=(32,), dtype=dtype, gate_std=0.3, w_std=0.18)
    lm = wl.make_toy_lm(cfg, V=V, L=2, seed=5, head_std=0.5)
    dev = ToyLMDevice.upload(lm, int8_head=True)
    q, scale = (t.cpu().double() for t in mm.quantize_rows(mm.to_device(lm.head, cfg)))
    rec = []
    run = Alg1Batch(dev, B, wl.make_prompt_tokens(3, 400, V), max_new=7, record=rec)
    for _ in range(30):
        run.step()
    gamma, kept, both = np.float32(cfg.gamma), [], [0, 0]
    for s, r in enumerate(rec):
        # logits: the codes' exact product; three roundings
        x, xs = (t.cpu().double() for t in mm.quantize_rows(r["x_head"].cuda()))
        z = (x @ q.t().contiguous()) * xs[:, None] * scale[None, :]
        got = torch.from_numpy(r["lm_logits"]).double()
        assert ((got - z).abs() <= z.abs() * (3 * 2.0 ** -24) * 1.0001).all(), s
        # confidence and token: of the stored logits
        p = torch.softmax(got, dim=1)
        assert ((torch.from_numpy(r["conf"]).double() - p.max(1).values).abs() <= 1e-5 * p.max(1).values).all()
        assert np.array_equal(r["top"], got.argmax(1).numpy())
        # the loop: a little pass with p <= gamma is run again in big mode and keeps nothing
        for b in range(B):
            if not r["big_in"][b] and not (r["conf"][b] > gamma):
                both[0] += 1
                if s + 1 < len(rec):
                    assert rec[s + 1]["big_in"][b] and rec[s + 1]["conf_in"][b] == r["conf"][b]
            else:
                both[1] += 1
                kept.append((r["seq_id"][b], float(p[b].max().log()), float(-(p[b] * torch.log(p[b].clamp_min(1e-300))).sum())))
    assert both[0] > 0 and both[1] > 0 and run.n_fallbacks == both[0] and run.n_accepted == both[1]
    # log p and entropy stay with the tokens, sequence by sequence
    order = {}
    for sid, logp, ent in kept:
        order.setdefault(sid, []).append((logp, ent))
    done = [(f[0], f[1], lp, en) for f, lp, en in zip(run.finished, run.finished_logp, run.finished_entropy)]
    done += [(run.seq_id[b], run.tokens[b], run.token_logp[b], run.token_entropy[b]) for b in range(B)]
    assert sum(len(d[2]) for d in done) == len(kept)
    for sid, tokens, lp, en in done:
        assert len(tokens) - 1 == len(lp) == len(en)
        if lp:
            want = order[sid]
            assert np.allclose(lp, [w[0] for w in want], rtol=1e-4, atol=1e-6) and np.allclose(en, [w[1] for w in want], rtol=1e-4, atol=1e-6)


def test_a_small_vocabulary_keeps_the_router_head():
    cfg = wl.LayerConfig(name="toy", T=1, H=64, E=8, I=48, k_big=4, k_little=2, dtype="bf16", gate_std=0.3, w_std=0.18)
    with pytest.raises(ValueError, match="256"):
        ToyLMDevice.upload(wl.make_toy_lm(cfg, V=257, L=1, seed=1))
    assert ToyLMDevice.upload(wl.make_toy_lm(cfg, V=256, L=1, seed=1)).int8_head is None
