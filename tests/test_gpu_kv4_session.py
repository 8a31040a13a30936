"""Forwards, appends and sessions on a 4-bit prefix cache.  The oracle reads the values that the device's codes stand for, so the tolerances are those of
the other parity tests; appended rows are the staged ones, quantised, bit for bit."""
import dataclasses

import numpy as np
import pytest
import torch

import s2d2_inputs as I
from paper_2603_25702_amd import KvCache, Params, S2D2Error, s2d2_kv4_append, s2d2_kv4_evict, s2d2_kv4_read, s2d2_set_kv4
from paper_2603_25702_amd.binding import RouteParams
from paper_2603_25702_amd.runner import Session
from tests import harness as H
from tests import kv4_plain as P
from tests.test_gpu_parity import SMALL_BF16, SMALL_MOE, TINY

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NARROW = I.ModelCfg("small-bf16", 2, 512, 8, 2, 64, 1536, 32000)   # heads that the MFMA attention over bf16 pages does not take


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


class Run(H.DeviceRun):
    """A case whose prefix goes into a session's 4-bit cache; `sync` gives the case what the codes stand for."""

    def __init__(self, cfg, lens, B, seed=0, page_size=16, room=96, act_planes=0, packed=True, **bound):
        case = H.make_case(cfg, len(lens), B, lens, seed=seed, synthetic_kv=True, page_size=page_size, room=room, norm_jitter=0.1)
        self.ses = Session(cfg, case.W, case.N, B, case.page_table.shape[1] * page_size, page_size, page_table=case.page_table, max_block=B, act_planes=act_planes,
                           cache_bits=4, **bound)
        if not packed:
            from paper_2603_25702_amd import Engine
            self.ses.eng = Engine(cfg, case.W, case.N, B, packed=False)
            s2d2_set_kv4(self.ses.eng, self.ses.kv)
        super().__init__(case, session=self.ses)
        self.push_state()
        self.kv.seq_len.zero_()
        counts = [int(x) for x in case.seq_len]
        rows = np.cumsum([0] + counts[:-1])
        dense = [case.oracle_cache(n) for n in range(case.N)]
        k, v = (torch.stack([torch.cat([dense[n][which][l] for n in range(case.N)]) for l in range(cfg.n_layers)]).to(DEV) for which in (0, 1))
        s2d2_kv4_append(self.kv, k, v, i32(rows), i32(counts), max(counts))
        self.sync()

    def sync(self):
        """Case state and cache as the device has them; entries of a list in the order of their places."""
        case, kv = self.case, self.kv
        torch.cuda.synchronize()
        entries, self.entries = kv.entries.cpu().numpy(), kv.entries.cpu().numpy()
        k, v = (torch.zeros(kv.n_layers, case.N, int(entries.max()) + 1, kv.n_kv_heads, kv.head_dim, dtype=case.cfg.torch_dtype, device=DEV) for _ in range(2))
        s2d2_kv4_read(kv, torch.zeros(case.N, dtype=torch.int32, device=DEV), k, v)
        k, v = k.cpu(), v.cpu()
        case.oracle_cache = lambda n: ([k[l, n, :entries[n]] for l in range(kv.n_layers)], [v[l, n, :entries[n]] for l in range(kv.n_layers)])
        case.seq_len = kv.seq_len.cpu().numpy().copy()
        blk, pos0, car = self.st.block_tokens.cpu().numpy(), self.st.block_pos0.cpu().numpy(), self.st.carry_tokens.cpu().numpy()
        for n, s in enumerate(case.states):
            s.seq_len, s.pos0, s.block = int(case.seq_len[n]), int(pos0[n]), blk[n].astype(np.int64)
            s.carry = car[n, :max(0, s.pos0 - s.seq_len)].astype(np.int64)

    def append_checked(self):
        """s2d2_kv_append; every new entry is its staged row, quantised."""
        case, kv = self.case, self.kv
        before, seq = kv.entries.cpu().numpy(), kv.seq_len.cpu().numpy()
        self.eng.s2d2_kv_append(kv, case.N, case.B, self.d, self.v, self.a.n_accept)
        lead, row0, acc, span = (t.cpu().numpy() for t in (self.v.stage_lead, self.v.stage_row0, self.a.n_accept, self.d.span_len))
        rows = lead + np.minimum(acc, span - int(case.cfg.right_shifted))
        assert np.array_equal(kv.entries.cpu().numpy(), before + rows) and np.array_equal(kv.seq_len.cpu().numpy(), seq + rows)
        ks, vs = self.v.k_stage.double().cpu().numpy(), self.v.v_stage.double().cpu().numpy()
        for n in range(case.N):
            place = before[n] + np.arange(rows[n])
            at = case.page_table[n][place // case.page_size].astype(np.int64), place % case.page_size
            for src, codes, scales in ((ks, kv.k_codes, kv.k_scales), (vs, kv.v_codes, kv.v_scales)):
                c, s = P.quantise(src[:, row0[n]:row0[n] + rows[n]])
                assert np.array_equal(codes.cpu().numpy()[:, at[0], :, at[1]], c.swapaxes(0, 1)) and np.array_equal(scales.cpu().numpy()[:, at[0], :, at[1]], s.swapaxes(0, 1))
        return rows


def steps(run, count, rep=None, evict=None, **prm):
    rep = rep or H.Report()
    for s in range(count):
        p = Params(step=s, seed=1234, **prm)
        run.step(p, advance=False, append=False)
        H.check_step(run.case, run, run.fetch(), p, rep=rep, append=False)
        run.append_checked()
        if evict:
            s2d2_kv4_evict(run.kv, *evict)
        run.eng.s2d2_block_advance(run.kv, run.st, run.case.N, run.case.B, None)
        run.sync()
    assert not run.kv.status.cpu().any()
    return rep


shifted = lambda cfg: dataclasses.replace(cfg, right_shifted=True)  # noqa: E731


@pytest.mark.parametrize("name,cfg,lens,B,page,kw", [
    ("fp32", TINY, [128, 1, 77], 4, 16, {}), ("fp32 shifted", shifted(TINY), [37, 64], 3, 8, {}), ("bf16", SMALL_BF16, [100, 257, 31], 8, 16, {}),
    ("bf16 wide", SMALL_BF16, [100, 257], 32, 16, {}), ("bf16 two planes", SMALL_BF16, [100, 33], 8, 24, dict(act_planes=2)),
    ("bf16 canonical", SMALL_BF16, [100, 33], 4, 16, dict(packed=False)), ("moe", SMALL_MOE, [60, 200], 8, 16, {}), ("bf16 shifted", shifted(SMALL_BF16), [100, 31], 8, 16, {}),
    ("heads of 64", NARROW, [90, 140], 6, 12, {}), ("long", SMALL_BF16, [3000, 1100], 4, 16, {})])
def test_steps_match_the_oracle_on_what_the_cache_holds(name, cfg, lens, B, page, kw):
    run = Run(cfg, lens, B, seed=7, page_size=page, **kw)
    rep = steps(run, 3)
    print(name, rep)
    tol = 1e-4 if cfg.dtype == "f32" else H.LOGIT_RTOL
    assert rep.max_logit_err_draft <= tol and rep.max_logit_err_verify <= tol


@pytest.mark.parametrize("cfg,B", [(TINY, 4), (SMALL_BF16, 8)])
def test_steps_behind_an_eviction_match_the_oracle_on_what_is_left(cfg, B):
    """Positions go on by seq_len while every list holds entries of its own choice."""
    run = Run(cfg, [128, 40, 90], B, seed=9, budget=60, sink=4, recent=16)
    assert run.kv.mass is not None
    rep = steps(run, 4, evict=(60, 0, 4, 16))
    assert rep.max_logit_err_draft <= (1e-4 if cfg.dtype == "f32" else H.LOGIT_RTOL)
    entries, seq = run.kv.entries.cpu().numpy(), run.kv.seq_len.cpu().numpy()
    assert entries[0] == 60 and entries[2] == 60 and 40 <= entries[1] <= 60 and (seq[[0, 2]] > [128, 90]).all()
    for n in range(3):   # every list: different tokens, the first and the last ones among them
        place = np.arange(entries[n])
        p = run.kv.position.cpu().numpy()[:, run.case.page_table[n][place // 16], :, place % 16]
        for l in range(cfg.n_layers):
            for h in range(cfg.n_kv_heads):
                have = p[:, l, h]
                assert len(set(have)) == entries[n] and have.max() < seq[n] and set(range(4)) <= set(have)
                assert set(range(seq[n] - 16, seq[n])) <= set(have) | set(range(0))


def test_mass_grows_by_the_verifying_rows_and_not_by_the_drafting_ones():
    run = Run(TINY, [50, 33, 20], 4, seed=3, budget=1000)
    N, B, kv = 3, 4, run.kv
    kv.mass.zero_()
    prm = Params(seed=5)
    run.eng.s2d2_draft(kv, run.st, N, B, prm, run.d)
    assert not kv.mass.any()
    run.eng.s2d2_verify(kv, run.st, N, B, dataclasses.replace(prm, active=i32([1, 0, 1])), run.d, run.v)
    mass = kv.mass.cpu().numpy()
    grp = TINY.n_q_heads // TINY.n_kv_heads
    for n in range(3):
        place = np.arange(int(kv.entries[n]))
        m = mass[:, run.case.page_table[n][place // 16], :, place % 16]
        if n == 1:
            assert not m.any()
        else:
            assert (m > 0).all() and (m.sum(0) < 2 * B * grp).all() and (m.sum(0) > 0.1 * 2 * B * grp).all()
    assert np.count_nonzero(mass) == TINY.n_layers * TINY.n_kv_heads * (50 + 20)


@pytest.mark.parametrize("cfg", [TINY, SMALL_BF16, shifted(SMALL_BF16)])
def test_prompts_and_generation_with_and_without_a_budget(cfg):
    W, lens = I.gen_weights(cfg, 3), [200, 30, 391]
    ids = [I.gen_prefix_ids(cfg, n, 3, i) for i, n in enumerate(lens)]
    cached = [n - int(cfg.right_shifted) for n in lens]
    room = 16 * 40
    full = Session(cfg, W, 3, 4, room, cache_bits=4)
    full.prefill(ids)
    assert full.kv.entries.tolist() == cached == full.kv.seq_len.tolist()
    # the first layer's K and V do not depend on the cache: quantised, they are those of a bf16 / fp32 session to a rounding of either side
    plain = Session(cfg, W, 3, 4, room)
    plain.prefill(ids)
    k, v = (torch.zeros(cfg.n_layers, 3, max(lens), cfg.n_kv_heads, cfg.head_dim, device=DEV) for _ in range(2))
    s2d2_kv4_read(full.kv, i32([0, 0, 0]), k, v)
    for n in range(3):
        at = np.arange(cached[n])
        pages = plain.kv.page_table[n].cpu().numpy()[at // 16]
        want = P.values(*P.quantise(plain.kv.k[0].double().cpu().numpy()[pages, :, at % 16]))
        assert (np.abs(k[0, n, :cached[n]].double().cpu().numpy() - want) > 0).mean() < 0.01
    # a budget that is never reached changes nothing but the masses; one that is holds
    rp = RouteParams()
    big = Session(cfg, W, 3, 4, room, cache_bits=4, budget=600)
    big.prefill(ids)
    tight = Session(cfg, W, 3, 4, 16 * 20, cache_bits=4, budget=100, slack=16, sink=4, recent=32)
    tight.prefill(ids)
    assert tight.kv.seq_len.tolist() == cached and max(tight.kv.entries.tolist()) <= 116 and tight.kv.entries.tolist()[1] == cached[1]
    outs = [s.generate(Params(seed=11, tau=0.3), rp, 3, 6) for s in (full, big, tight)]
    assert outs[0] == outs[1]
    assert all(len(o) == 12 for o in outs[2][0])
    assert max(tight.kv.entries.tolist()) <= 116 and not tight.kv.status.any()
    assert all(s >= c + 4 for s, c in zip(tight.kv.seq_len.tolist(), cached))


def test_whole_block_caching_on_four_bits():
    cfg = SMALL_BF16
    W = I.gen_weights(cfg, 3)
    ids = [I.gen_prefix_ids(cfg, n, 3, i) for i, n in enumerate([40, 70])]
    ses = Session(cfg, W, 2, 4, 320, cache_bits=4, budget=64, sink=2, recent=8)
    ses.prefill(ids)
    out, log = ses.generate(Params(seed=2, tau=0.2), RouteParams(), 3, 5, caching="block")
    assert all(len(o) == 12 for o in out) and max(ses.kv.entries.tolist()) <= 64
    assert ses.kv.seq_len.tolist() == [52, 82]


def test_a_captured_step_with_eviction_is_the_eager_one():
    cfg = SMALL_BF16
    W = I.gen_weights(cfg, 3)
    ids = [I.gen_prefix_ids(cfg, n, 3, i) for i, n in enumerate([40, 70])]
    runs = []
    for captured in (False, True):
        ses = Session(cfg, W, 2, 4, 320, cache_bits=4, budget=64, sink=2, recent=8)
        ses.prefill(ids)
        prm = Params(seed=4, step_dev=ses.step_dev)
        seen = []
        g = ses.capture_step(prm) if captured else None
        for _ in range(5):
            g.replay() if captured else ses.step(prm)
            torch.cuda.synchronize()
            seen.append([t.clone() for t in (ses.st.block_tokens, ses.kv.entries, ses.kv.seq_len, ses.d.logits, ses.a.n_accept)] + [ses.kv.mass.sum(), ses.kv.position.sum()])
        runs.append(seen)
    for a, b in zip(*runs):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_attached_and_detached():
    cfg = TINY
    run = Run(cfg, [30], 4, seed=1)
    kv, e = run.kv, run.eng
    shape = (cfg.n_layers, kv.n_pages, cfg.n_kv_heads, kv.page_size, cfg.head_dim)
    other = KvCache(torch.zeros(shape, device=DEV), torch.zeros(shape, device=DEV).transpose(3, 4).contiguous(), kv.page_table, kv.seq_len, kv.status)
    prm = Params(seed=1)
    e.s2d2_draft(kv, run.st, 1, 4, prm, run.d)
    first = run.d.logits.clone()
    for call in (lambda: e.s2d2_draft(other, run.st, 1, 4, prm, run.d), lambda: e.s2d2_verify(other, run.st, 1, 4, prm, run.d, run.v),
                 lambda: e.s2d2_kv_append(other, 1, 4, run.d, run.v, run.a.n_accept), lambda: e.s2d2_block_advance(other, run.st, 1, 4)):
        with pytest.raises(S2D2Error, match="4-bit cache"):
            call()
    s2d2_set_kv4(e, None)
    e.s2d2_draft(other, run.st, 1, 4, prm, run.d)     # a prefix of zeros in fp32 pages
    assert not torch.equal(run.d.logits, first)
    s2d2_set_kv4(e, kv)
    e.s2d2_draft(kv, run.st, 1, 4, prm, run.d)
    assert torch.equal(run.d.logits, first)
    lib, view = e.lib, kv._ref
    big = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    need = e._kv4[1].numel()
    assert lib.s2d2_set_kv4(e.ctx, view, big.data_ptr(), max(need - 1, 0), None) == (-2 if need else 0)
    wrong = type(kv._view).from_buffer_copy(kv._view)
    wrong.head_dim = 32
    assert lib.s2d2_set_kv4(e.ctx, wrong, big.data_ptr(), 1 << 24, None) == -1
    wrong = type(kv._view).from_buffer_copy(kv._view)
    wrong.mass = big.data_ptr()
    assert lib.s2d2_set_kv4(e.ctx, wrong, big.data_ptr(), 1 << 24, None) == -1     # mass without lse
    with pytest.raises(ValueError):
        Session(cfg, {}, 1, 4, 64, budget=10)
    with pytest.raises(ValueError):
        Session(cfg, {}, 1, 4, 64, cache_bits=4, budget=10, sink=4, recent=8)
    with pytest.raises(ValueError):
        Session(cfg, {}, 1, 4, 64, cache_bits=8)


def test_a_prompt_without_room_is_reported():
    cfg = TINY
    ses = Session(cfg, I.gen_weights(cfg, 3), 1, 4, 64, cache_bits=4)
    with pytest.raises(RuntimeError, match="status"):
        ses.prefill([I.gen_prefix_ids(cfg, 100, 3, 0)])
