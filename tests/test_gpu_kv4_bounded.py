"""Sessions on a bounded 4-bit cache: what the defaults keep, sessions that go on after a lack of room, prompts in the room that is promised, fresh blocks behind
a cache that was cut, streams."""
import numpy as np
import pytest
import torch

import s2d2_inputs as I
from paper_2603_25702_amd import Params, s2d2_set_kv4
from paper_2603_25702_amd.binding import RouteParams
from paper_2603_25702_amd.runner import Session
from tests.test_gpu_parity import SMALL_BF16, TINY

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def prompts(cfg, lens):
    return [I.gen_prefix_ids(cfg, n, 3, i) for i, n in enumerate(lens)]


def positions(kv, n):
    """[layers, entries, KV heads]"""
    place = np.arange(int(kv.entries[n]))
    return kv.position.cpu().numpy()[:, kv.page_table[n].cpu().numpy()[place // kv.page_size], :, place % kv.page_size].transpose(1, 0, 2)


# ---- what the defaults keep ----

@pytest.mark.parametrize("cfg,budget", [(TINY, 100), (SMALL_BF16, 60), (TINY, 16)])
def test_new_tokens_outlive_their_append_at_the_defaults(cfg, budget):
    """Once the budget is full, the tokens of a step are there at the next step's draft, in every list; and after many steps a part of the budget is theirs."""
    B = 4
    ses = Session(cfg, I.gen_weights(cfg, 3), 2, B, 512, cache_bits=4, budget=budget)
    ses.prefill(prompts(cfg, [391, 120]))
    kv = ses.kv
    assert kv.entries.tolist() == [budget, budget]
    grown = [0, 0]
    for step in range(30):
        before = kv.seq_len.tolist()
        ses.step(Params(seed=1, step=step, tau=0.0))
        after = kv.seq_len.tolist()
        for n in range(2):
            p = positions(kv, n)
            assert p.shape[1] == budget
            new = set(range(before[n], after[n]))
            grown[n] += len(new)
            for l in range(cfg.n_layers):
                for h in range(cfg.n_kv_heads):
                    have = set(p[l, :, h])
                    assert len(have) == budget and new <= have, (step, n, l, h)
    assert min(grown) > 15
    for n, prompt in enumerate((391, 120)):
        assert ((positions(kv, n) >= prompt).sum(1) >= min(grown[n], (budget - 4) // 2)).all()


# ---- a session that once had no room ----

def test_a_prompt_that_fits_after_one_that_did_not():
    cfg = TINY
    ses = Session(cfg, I.gen_weights(cfg, 3), 1, 4, 64, cache_bits=4)
    good = prompts(cfg, [30])
    fresh = Session(cfg, I.gen_weights(cfg, 3), 1, 4, 64, cache_bits=4)
    fresh.prefill(good)
    for _ in range(2):
        with pytest.raises(RuntimeError, match="status"):
            ses.prefill(prompts(cfg, [100]))
        ses.prefill(good)
        assert ses.kv.entries.tolist() == [30] == ses.kv.seq_len.tolist() and not ses.kv.status.any()
        assert ses.generate(Params(seed=3, tau=0.3), RouteParams(), 1, 5) == fresh.generate(Params(seed=3, tau=0.3), RouteParams(), 1, 5)
        fresh.prefill(good)
    # a sequence that ran out of room while it was generated
    with pytest.raises(RuntimeError, match="status"):
        ses.prefill(prompts(cfg, [60]))
        ses.generate(Params(seed=3, tau=0.0), RouteParams(), 4, 5)
    ses.prefill(good)
    assert ses.kv.entries.tolist() == [30]


def test_a_prompt_of_one_token_after_a_lack_of_room():
    """A right-shifted model caches nothing of it: no chunk, no room needed."""
    import dataclasses
    cfg = dataclasses.replace(TINY, right_shifted=True)
    ses = Session(cfg, I.gen_weights(cfg, 3), 1, 4, 64, cache_bits=4)
    with pytest.raises(RuntimeError, match="status"):
        ses.prefill(prompts(cfg, [100]))
    ses.prefill(prompts(cfg, [1]))
    assert ses.kv.entries.tolist() == [0] == ses.kv.seq_len.tolist()
