"""The mass of a session's entries against the definition in 64 bits, in the first layer, whose queries and keys the tokens alone give: every row of a
forward gives its softmax weights to the cached entries and to the window rows it sees, and a row that is appended brings along what its window gave it.

Error bound.  A projected value is a sum of d_model products in 32 bits of inputs that are off by a few roundings: (d_model + 16) * 2^-24 of the sum of their
magnitudes, the rotation adds an angle of at most 512 rounded to 32 bits, 2^-15.  A score is then off by scale * sum(|q| ek + |k| eq), a weight relative to its row's sum by twice that."""
import dataclasses

import numpy as np
import pytest
import torch

import s2d2_inputs as I
from oracle import s2d2_oracle as O
from paper_2603_25702_amd import Params, s2d2_kv4_read, s2d2_set_kv4
from paper_2603_25702_amd.runner import Session
from tests.test_gpu_kv4_session import Run, i32
from tests.test_gpu_parity import SMALL_BF16, TINY

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def first_layer(cfg, W, tokens, pos):
    """Queries and keys of the first layer, and the bounds of their errors."""
    a = O.rmsnorm(O.take_rows(W["embed"], tokens), O.f64(W["l0.norm1"]), cfg.rms_eps)
    w = O.f64(W["l0.wqkv"])[: (cfg.n_q_heads + cfg.n_kv_heads) * cfg.head_dim]
    x, e = a @ w.T, np.abs(a) @ np.abs(w).T * ((cfg.d_model + 16) * 2.0 ** -24 + 2.0 ** -15)
    x, e = (t.reshape(len(tokens), -1, cfg.head_dim) for t in (x, e))
    e = e + np.roll(e, cfg.head_dim // 2, -1)
    x = O.rope(x, np.asarray(pos), cfg.rope_theta)
    return (x[:, :cfg.n_q_heads], e[:, :cfg.n_q_heads]), (x[:, cfg.n_q_heads:], e[:, cfg.n_q_heads:])


def given(cfg, W, tokens, pos, vis, cached):
    """What the rows of one window give [cached entries and window rows, KV heads] in the first layer, and the bound of its error."""
    (q, eq), (k, ek) = first_layer(cfg, W, tokens, pos)
    n, s, grp, scale = len(tokens), len(cached), cfg.n_q_heads // cfg.n_kv_heads, cfg.head_dim ** -0.5
    out, off = np.zeros((s + n, cfg.n_kv_heads)), np.zeros((s + n, cfg.n_kv_heads))
    for h in range(cfg.n_q_heads):
        g = h // grp
        keys, ekeys = np.concatenate((cached[:, g], k[:, g])), np.concatenate((np.zeros_like(cached[:, g]), ek[:, g]))
        score = np.where(np.concatenate((np.ones((n, s), bool), vis), 1), scale * (q[:, h] @ keys.T), -np.inf)
        err = scale * (np.abs(q[:, h]) @ ekeys.T + eq[:, h] @ np.abs(keys).T)
        p = O.softmax_rows(score)
        out[:, g] += p.sum(0)
        off[:, g] += (p * (err + err.max(1, keepdims=True))).sum(0)
    return out, 1.5 * off + 1e-5 * out   # (second order; exponentials, sums, the rounding of lse)


def cached_keys(kv, most):
    k, v = (torch.zeros(kv.n_layers, kv.N, most, kv.n_kv_heads, kv.head_dim, device=DEV) for _ in range(2))
    s2d2_kv4_read(kv, torch.zeros(kv.N, dtype=torch.int32, device=DEV), k, v)
    return k[0].double().cpu().numpy()


def masses(kv, n, layer=0):
    place = np.arange(int(kv.entries[n]))
    pages = kv.page_table[n].cpu().numpy()[place // kv.page_size]
    return kv.mass.double().cpu().numpy()[layer, pages, :, place % kv.page_size]   # [entries, KV heads]


def test_a_prompt_s_rows_are_weighed_by_those_that_see_them():
    """Chunks of a prompt: rows of a later chunk see the entries of the earlier ones as they are cached."""
    cfg, lens = TINY, [200, 37, 100]
    W = I.gen_weights(cfg, 3)
    W["l0.wqkv"] = W["l0.wqkv"] * 3   # (weights that differ)
    ids = [I.gen_prefix_ids(cfg, n, 3, i) for i, n in enumerate(lens)]
    ses = Session(cfg, W, 3, 4, 512, cache_bits=4, budget=400)
    ses.prefill(ids)
    keys = cached_keys(ses.kv, 200)
    for n, L in enumerate(lens):
        want, off = np.zeros((L, cfg.n_kv_heads)), np.zeros((L, cfg.n_kv_heads))
        for at in range(0, L, 100):   # two equal chunks
            to = min(L, at + 100)
            m, e = given(cfg, W, ids[n][at:to], np.arange(at, to), O.causal_mask(to - at), keys[n, :at])
            want[:to] += m
            off[:to] += e
        got = masses(ses.kv, n)
        assert (np.abs(got - want) <= off).all(), (n, np.abs(got - want).max(), (off / want).max())
        assert (off < 0.05 * want).mean() > 0.9
    for l in range(cfg.n_layers):   # every row and head of a group gives 1 in all
        for n, L in enumerate(lens):
            assert np.allclose(masses(ses.kv, n, l).sum(0), L * cfg.n_q_heads // cfg.n_kv_heads, rtol=2.0 ** -14)


@pytest.mark.parametrize("cfg", [SMALL_BF16, dataclasses.replace(SMALL_BF16, right_shifted=True)])
@pytest.mark.parametrize("kw", [{}, dict(act_planes=2), dict(act_planes=1), dict(packed=False)])
def test_every_row_of_a_bf16_prompt_gives_its_heads_weight(cfg, kw):
    """bf16 rows in every operand mode: what the rows of a prompt give sums up to their number, up to the roundings of lse and of the sums; a prompt of
    several tiles of rows and keys."""
    lens, kw = [150, 33], dict(kw)
    W = I.gen_weights(cfg, 3)
    packed = kw.pop("packed", True)
    ses = Session(cfg, W, 2, 4, 512, cache_bits=4, budget=400, **kw)
    if not packed:
        from paper_2603_25702_amd import Engine, s2d2_set_kv4
        ses.eng = Engine(cfg, W, 2, 64, packed=False)
        s2d2_set_kv4(ses.eng, ses.kv)
    ses.prefill([I.gen_prefix_ids(cfg, n, 3, i) for i, n in enumerate(lens)])
    for n, L in enumerate(lens):
        L -= int(cfg.right_shifted)
        for l in range(cfg.n_layers):
            m = masses(ses.kv, n, l)
            assert (m > 0).all() and np.allclose(m.sum(0), L * cfg.n_q_heads // cfg.n_kv_heads, rtol=2.0 ** -14)
            # the last row is seen by itself only, the first by all
            assert (m[-1] <= cfg.n_q_heads // cfg.n_kv_heads).all() and (m[0] > m[-1]).all()


def test_accepted_rows_bring_what_their_verification_gave_them():
    cfg, B = TINY, 4
    run = Run(cfg, [50, 33, 20], B, seed=3, budget=1000)
    kv = run.kv
    for step in range(4):   # later windows have pending rows in front; of the last one every drafted row is appended, whatever was accepted
        kv.mass.zero_()
        entries = kv.entries.cpu().numpy()
        keys = cached_keys(kv, int(entries.max()) + 1)
        run.step(Params(step=step, seed=5, tau=0.02), advance=False, append=False)
        windows = [O.verify_window(s, run.d.xhat[n].cpu().numpy(), cfg.mask_id) for n, s in enumerate(run.case.states)]
        if step == 3:
            run.a.n_accept.copy_(run.d.span_len)
        rows = run.append_checked()
        assert step == 0 or (rows > 0).any()
        for n, w in enumerate(windows):
            if w.L == 0:
                continue
            want, off = given(cfg, run.case.W, w.tokens, w.pos, w.vis, keys[n, :entries[n]])
            got, here = masses(kv, n), int(entries[n] + rows[n])
            assert got.shape[0] == here
            assert (np.abs(got - want[:here]) <= off[:here]).all(), (step, n)
            assert (got[entries[n]:] > 0).all()
        run.eng.s2d2_block_advance(kv, run.st, 3, B, None)
        run.sync()


def test_entries_of_a_later_chunk_win_by_their_weight():
    """A prompt of three chunks that is cut to a budget after each, nothing protected: what is left is what the definition keeps, list by list."""
    cfg, budget, T = TINY, 60, 128
    W = I.gen_weights(cfg, 5)
    W["l0.wqkv"] = W["l0.wqkv"] * 4   # (by the definition 8 places go to later chunks; of weights that are not so peaked, none)
    ids = I.gen_prefix_ids(cfg, 3 * T, 4, 0)
    ses = Session(cfg, W, 1, 4, 512, cache_bits=4, budget=budget, sink=0, recent=0)
    kv, e = ses.kv, ses.eng
    tok = torch.from_numpy(np.asarray(ids, np.int32)).to(DEV).view(1, -1)
    later = 0
    for c in range(3):
        held = int(kv.entries[0])
        place = np.arange(held)
        keys, before = cached_keys(kv, held + 1)[0, :held], masses(kv, 0)
        old = kv.position.cpu().numpy()[0, kv.page_table[0].cpu().numpy()[place // 16], :, place % 16]
        e.s2d2_prefill(kv, 1, T, tok, c * T, i32([T]), ses.v.k_stage, ses.v.v_stage)
        want, off = given(cfg, W, ids[c * T:(c + 1) * T], np.arange(c * T, (c + 1) * T), O.causal_mask(T), keys)
        want[:held] += before
        assert (np.abs(masses(kv, 0) - want) <= off + 1e-6 * want).all(), c
        ses._evict()
        assert kv.entries.tolist() == [budget]
        place = np.arange(budget)
        now = kv.position.cpu().numpy()[0, kv.page_table[0].cpu().numpy()[place // 16], :, place % 16]
        for h in range(cfg.n_kv_heads):
            position = np.concatenate((old[:, h], np.arange(c * T, (c + 1) * T)))
            border = np.sort(want[:, h])[-budget]
            sure, never = want[:, h] - off[:, h] > border + off[:, h].max(), want[:, h] + off[:, h] < border - off[:, h].max()
            assert set(position[sure]) <= set(now[:, h]) and not set(position[never]) & set(now[:, h])
            later += int((now[:, h] >= T).sum())
    assert later > 0


def test_rows_that_no_forward_weighed_since_the_cache_was_attached_bring_nothing():
    cfg = TINY
    run = Run(cfg, [40, 20], 4, seed=3, budget=1000)
    run.step(Params(seed=5), advance=False, append=False)
    run.a.n_accept.copy_(run.d.span_len)
    s2d2_set_kv4(run.eng, run.kv)
    assert (run.append_checked() > 0).all()
    for n, s in enumerate((40, 20)):
        m = masses(run.kv, n)
        assert (m[:s] > 0).all() and (m[s:] == 0).all()
