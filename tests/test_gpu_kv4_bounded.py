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


# ---- room ----

@pytest.mark.parametrize("budget,slack,length", [(100, 8, 391), (40, 0, 200), (16, 0, 193)])
def test_prompts_of_any_length_in_the_room_that_is_promised(budget, slack, length):
    """Room for budget + slack entries and the rows of one append: chunks of a prompt are no longer than that."""
    cfg, B = TINY, 4
    ses = Session(cfg, I.gen_weights(cfg, 3), 2, B, budget + slack + 2 * B, page_size=4, cache_bits=4, budget=budget, slack=slack)
    ses.prefill(prompts(cfg, [length, 20]))
    assert ses.kv.seq_len.tolist() == [length, 20] and ses.kv.entries.tolist()[0] <= budget + slack
    out, _ = ses.generate(Params(seed=2, tau=0.2), RouteParams(), 3, 5)
    assert all(len(o) == 12 for o in out)


def test_chunks_stay_as_they_are_where_there_is_room():
    """Chunks of 131 of a prompt of 391 go into 240 places with a budget of 100: the entries in front of a chunk are the budget, not what it may grow to."""
    cfg = TINY
    W, ids = I.gen_weights(cfg, 3), prompts(cfg, [391])
    wide, tight = (Session(cfg, W, 1, 4, room, cache_bits=4, budget=100, slack=16) for room in (640, 240))
    calls = []
    for ses in (wide, tight):
        call, here = ses.eng.s2d2_prefill, []
        ses.eng.s2d2_prefill = lambda kv, N, T, *a, call=call, here=here: (here.append(T), call(kv, N, T, *a))
        ses.prefill(ids)
        calls.append(here)
    assert calls == [[131, 131, 131]] * 2
    assert np.array_equal(positions(wide.kv, 0), positions(tight.kv, 0))


# ---- fresh blocks ----

def test_fresh_blocks_behind_a_cache_that_was_cut():
    cfg = SMALL_BF16
    lens = [200, 30]
    ses = Session(cfg, I.gen_weights(cfg, 3), 2, 4, 320, cache_bits=4, budget=64)
    ses.prefill(prompts(cfg, lens))
    prm, kv = Params(seed=1), ses.kv
    ses.eng.s2d2_draft(kv, ses.st, 2, 4, prm, ses.d)
    want = ses.d.logits.clone()
    ses.reset_blocks(lens)                       # where they are already
    assert kv.entries.tolist() == [64, 30] and kv.seq_len.tolist() == lens
    ses.eng.s2d2_draft(kv, ses.st, 2, 4, prm, ses.d)
    assert torch.equal(ses.d.logits, want)
    for step in range(4):
        ses.step(Params(seed=1, step=step, tau=0.0))
    now, held = kv.seq_len.tolist(), kv.entries.tolist()
    assert held[0] == 64 and now[0] > 200 and held[1] == now[1] > 30
    with pytest.raises(ValueError, match="evicted"):
        ses.reset_blocks(lens)                   # which of the first sequence's entries lie before 200 differs from list to list
    assert kv.seq_len.tolist() == now and kv.entries.tolist() == held
    ses.reset_blocks([now[0], 25])               # the second one's are in order: back to 25
    assert kv.seq_len.tolist() == [now[0], 25] and kv.entries.tolist() == [64, 25]
    ses.prefill(prompts(cfg, lens))              # and from the start again
    ses.eng.s2d2_draft(kv, ses.st, 2, 4, prm, ses.d)
    assert torch.equal(ses.d.logits, want)


# ---- streams ----

def test_eviction_runs_on_the_stream_of_the_forwards():
    """Sessions that are made under one stream and stepped under another."""
    cfg = SMALL_BF16
    W, ids, runs = I.gen_weights(cfg, 3), prompts(cfg, [200, 90]), []
    side = torch.cuda.Stream()
    for made, stepped in ((None, None), (None, side), (side, None)):
        torch.cuda.synchronize()
        with torch.cuda.stream(made):
            ses = Session(cfg, W, 2, 4, 320, cache_bits=4, budget=64, recent=8)
            ses.prefill(ids)
        torch.cuda.synchronize()
        seen = []
        with torch.cuda.stream(stepped):
            for step in range(6):
                with torch.cuda.stream(made or torch.cuda.default_stream()):
                    torch.cuda._sleep(1_000_000)   # (what does not wait for the forwards is ahead of them)
                ses.step(Params(seed=4, step=step))
            torch.cuda.synchronize()
            seen = [t.clone() for t in (ses.st.block_tokens, ses.kv.entries, ses.kv.seq_len, ses.d.logits, ses.kv.mass, ses.kv.position)]
        torch.cuda.synchronize()
        runs.append(seen)
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


def test_the_scratch_of_a_detached_cache_is_not_handed_out_while_it_is_used():
    cfg = SMALL_BF16
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        ses = Session(cfg, I.gen_weights(cfg, 3), 1, 4, 4096, cache_bits=4, budget=64)
    torch.cuda.synchronize()
    with torch.cuda.stream(None):
        s2d2_set_kv4(ses.eng, ses.kv)            # (a scratch of the default stream's memory, used on the engine's)
        torch.cuda.synchronize()
        old = [t.data_ptr() for t in ses.eng._kv4[1:]]
        sizes = [t.numel() * t.element_size() for t in ses.eng._kv4[1:]]
        with torch.cuda.stream(side):
            torch.cuda._sleep(50_000_000)        # the engine's stream is busy for a while
        s2d2_set_kv4(ses.eng, None)
        new = [torch.empty(s, dtype=torch.uint8, device=DEV) for s in sizes]
        assert not set(old) & {t.data_ptr() for t in new}
    torch.cuda.synchronize()
