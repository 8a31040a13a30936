"""Attention over the 4-bit cache, and the weights its entries gather, against the definition in 64 bits.

Error bounds.  A score is a sum of D exact products in 32 bits: off by at most D * 2^-24 * sum |q||k|, times scale; scaling and exponent add
4 * 2^-24 of the same magnitude and 2^-21 (the exponential's last bits).  A weight relative to its row's sum is then off by twice that.  Of bf16 rows the
weights are rounded to half (2^-11 each; 2^-32 of the largest below 2^-21 of it) and the output to bf16 (2^-8); of fp32 rows two half planes keep 2^-22,
window values three bf16 planes each; sums of n terms in 32 bits add n * 2^-24 at most, sqrt(n) * 2^-24 * 8 is allowed.  All of it relative to sum p |v|."""
import math

import numpy as np
import pytest
import torch

from paper_2603_25702_amd import Kv4Rows, s2d2_kv4_attention, s2d2_kv4_attention_bytes, s2d2_kv4_weigh

from . import kv4_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(np.asarray(v), dtype=torch.int32, device=DEV)


def windows(kind, counts, gap=0):
    """row0, lo, hi, rows of packed windows, `gap` rows of nobody between them."""
    row0, r, lo, hi = [], gap, [], []
    lo, hi = [0] * gap, [0] * gap
    for c in counts:
        row0.append(r)
        half = c // 2
        for t in range(c):
            lo.append(r)
            hi.append(r + c if kind == "block" else r + t - half if kind == "verify" and t >= half else r + t + 1)
        r += c + gap
        lo += [0] * gap
        hi += [0] * gap
    return row0, lo, hi, max(r, 1)


class Case:
    def __init__(self, lens, counts, hq, hkv, d, page, dtype, kind, layers=1, layer=0, gap=0, T=None, seed=0, pad=0, lse=True, qscale=1.0, cache=None):
        self.cache = cache or P.Cache(lens, hkv, d, page, layers=layers, seed=seed)
        self.counts, self.layer, self.kind, self.dtype = counts, layer, kind, dtype
        self.row0, lo, hi, rows = windows(kind, counts, gap)
        gen = torch.Generator().manual_seed(seed)
        full = lambda heads: (torch.randn(rows, heads + pad, d, generator=gen) * qscale).to(dtype).to(DEV)[:, :heads]  # noqa: E731
        self.q, self.k, self.v = full(hq), None, None
        if kind != "none":
            self.k, self.v = full(hkv), full(hkv)
        self.lo, self.hi = (lo, hi) if kind in ("block", "verify") else (None, None)
        self.out = torch.full((rows, hq + pad, d), 55.0, dtype=dtype, device=DEV)[:, :hq]
        self.lse = torch.full((rows, hq), 55.0, device=DEV) if lse else None
        self.scale, self.T = d ** -0.5, T or max(max(counts), 1)
        self.make()

    def make(self):
        self.rows = Kv4Rows(self.q, i32(self.row0), i32(self.counts), self.T, self.scale, out=self.out, lse=self.lse, k=self.k, v=self.v,
                            lo=None if self.lo is None else i32(self.lo), hi=None if self.hi is None else i32(self.hi))
        need = s2d2_kv4_attention_bytes(self.cache.c, len(self.counts), self.T, self.q.shape[1])
        self.scratch = torch.full((max(need, 16),), 255, dtype=torch.uint8, device=DEV)   # (its contents do not matter: NaN)

    def run(self, **kw):
        s2d2_kv4_attention(self.cache.c, self.layer, self.rows, self.scratch, **kw)
        return self

    def want(self):
        f = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        return P.attention(self.cache, self.layer, f(self.q), self.row0, self.counts, self.scale, f(self.k), f(self.v), self.lo, self.hi)

    def check(self, want=None):
        out, lse, absout, most = want or self.want()
        mine = np.zeros(out.shape[0], bool)
        for r0, c in zip(self.row0, self.counts):
            mine[r0:r0 + c] = True
        d, n = out.shape[2], max(self.cache.lens + [1]) + self.T
        rel = 2 * (most[..., None] * (d + 4) * 2.0 ** -24 + 2.0 ** -21) + 8 * math.sqrt(n) * 2.0 ** -24
        rel += 2.0 ** -11 if self.dtype == torch.bfloat16 else 2.0 ** -21
        got = self.out.double().cpu().numpy()
        assert np.array_equal(np.isnan(got[mine]), np.isnan(out[mine]))
        # the term of the weights far below the largest (it counts where the large ones meet a value of 0): half has a step of 2^-24 there, an error of
        # 2^-25 a key, the largest weight is at least 2^7 by the choice of the reference: 2^-32 of the sum for every key, times its |v|
        vmost = max([np.abs(x).max() for x in self.cache.v[self.layer] if x.size and np.isfinite(x).any()] + [1.0])
        vmost = vmost if np.isfinite(vmost) else 1e3
        room = rel * absout + (2.0 ** -8 * np.abs(out) if self.dtype == torch.bfloat16 else 0) + n * 2.0 ** -32 * vmost
        off = np.abs(got - out)[mine]
        assert not (off > room[mine]).any(), f"worst {np.nanmax(off / room[mine]):.2f} of the bound"
        assert (got[~mine] == 55).all()
        if self.lse is not None:
            got = self.lse.double().cpu().numpy()
            assert np.array_equal(np.isnan(got[mine]), np.isnan(lse[mine]))
            assert np.array_equal(np.isinf(got[mine]), np.isinf(lse[mine]))
            fin = np.isfinite(lse) & mine[:, None]
            room = most * (d + 4) * 2.0 ** -24 + 2.0 ** -21 + 8 * math.sqrt(n) * 2.0 ** -24 + np.abs(lse) * 2.0 ** -23
            assert not (np.abs(got - lse)[fin] > room[fin]).any()
            assert (got[~mine] == 55).all()


BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hkv,d,page", [(4, 2, 32, 16), (7, 1, 64, 3), (8, 8, 128, 16), (10, 2, 256, 100), (32, 4, 128, 1)])
@pytest.mark.parametrize("kind", ["causal", "block", "verify", "none"])
def test_every_mask_type_and_head_layout(dtype, hq, hkv, d, page, kind):
    lens = [0, 1, 31, 32, 33, 95, 256, 300]
    Case(lens, [3, 1, 6, 0, 9, 2, 34, 5], hq, hkv, d, page, dtype, kind, layers=2, layer=1, gap=1, seed=d + page).run().check()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("lens,counts", [([1024], [1]), ([1025], [1]), ([992], [33]), ([8191, 0, 1, 2049, 4096], [2, 3, 1, 0, 1]), ([20000], [1]),
                                         ([1023, 1024, 1025, 3000], [40, 1, 64, 7])])
def test_long_caches_are_split_and_joined(dtype, lens, counts):
    Case(lens, counts, 8, 2, 64, 16, dtype, "block", seed=len(lens)).run().check()


def test_many_sequences_and_wide_windows():
    rng = np.random.default_rng(3)
    lens, counts = [int(x) for x in rng.integers(0, 200, 130)], [int(x) for x in rng.integers(0, 4, 130)]
    Case(lens, counts, 4, 2, 32, 8, BF, "causal").run().check()
    Case([500, 40], [192, 150], 8, 2, 64, 16, BF, "block").run().check()
    Case([500, 40], [70, 192], 6, 2, 64, 16, F32, "verify").run().check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_rows_any_distance_apart_a_wider_bound_and_no_lse(dtype):
    Case([50, 7], [3, 4], 4, 2, 64, 16, dtype, "block", pad=3, T=40, lse=False).run().check()
    Case([50, 7], [3, 4], 4, 2, 64, 16, dtype, "none", pad=1).run().check()


def test_counts_and_rows_out_of_range():
    case = Case([40, 50, 60, 70, 80], [2, 3, 1, 2, 4], 4, 2, 64, 16, BF, "causal")
    rows = case.q.shape[0]
    case.row0 = [0, 2, rows - 1, -1, 6]
    given = [-3, 99, 2, 2, 2]                 # below zero; cut to T; leaves the rows behind, in front; as it is
    case.counts = given
    case.make()
    case.counts = [0, 4, 0, 0, 2]
    case.T = 4
    case.run().check()


def test_entries_and_pages_out_of_range_are_read_as_the_nearest():
    case = Case([40, 50, 33], [1, 1, 2], 4, 2, 64, 16, BF, "none")
    cap = case.cache.table.shape[1] * 16
    c = case.cache
    c.c.entries[0] = -4
    c.lens[0], c.k[0][0], c.v[0][0] = 0, c.k[0][0][:0], c.v[0][0][:0]
    c.c.entries[1] = 10 ** 9                  # the whole table: 50 entries, then what stands in its pages
    pages, slots = c.places(1, cap)
    pages = np.clip(pages, 0, c.c.n_pages - 1)
    for name, store in (("k", c.k), ("v", c.v)):
        codes, scales = getattr(c.c, name + "_codes")[0].cpu().numpy(), getattr(c.c, name + "_scales")[0].cpu().numpy()
        np.minimum(scales, 140, out=scales)
        getattr(c.c, name + "_scales")[0].copy_(torch.from_numpy(scales))
        store[0][1] = P.values(codes[pages, :, slots], scales[pages, :, slots])
        store[0][2] = P.values(codes[c.places(2, 33)[0], :, c.places(2, 33)[1]], scales[c.places(2, 33)[0], :, c.places(2, 33)[1]])
    c.lens[1] = cap
    case.run().check()


@pytest.mark.parametrize("dtype", [BF, F32])
def test_masked_places_may_hold_anything(dtype):
    """NaN and infinities in window rows that a row does not see, in rows of nobody, in its own row's neighbours; noise behind the entries (every case has it)."""
    case = Case([40, 0, 70], [6, 6, 6], 4, 2, 64, 16, dtype, "verify", gap=2)
    for r, what in ((case.row0[0] + 5, math.nan), (case.row0[1] + 5, math.inf), (case.row0[2] + 2, -math.inf), (0, math.nan)):
        case.k[r] = what
        case.v[r, 1, 3] = what
    case.make()
    case.run()
    with np.errstate(all="ignore"):
        want = case.want()
    out, lse = want[0], want[1]
    got = case.out.double().cpu().numpy()
    # the last [MASK] copies see themselves only; drafted row 2 of the third sequence is seen by itself; copies 3 .. see what is left of them
    for r0, hit in ((case.row0[0], [5]), (case.row0[1], [5]), (case.row0[2], [2])):
        for t in range(6):
            assert np.isnan(got[r0 + t]).any() == (t in hit), (r0, t)
    for t in (out, lse, want[2], want[3]):
        t[np.isnan(got).any((1, 2))] = np.nan
    bad = np.isnan(got).any((1, 2))
    case.out[torch.from_numpy(bad).to(DEV)] = math.nan
    case.lse[torch.from_numpy(bad).to(DEV)] = math.nan
    case.check((out, lse, want[2], want[3]))


def test_a_group_that_reads_as_nan_is_nan_for_those_who_see_it():
    case = Case([40, 70], [2, 2], 4, 2, 64, 16, BF, "causal")
    c = case.cache
    (p,), (s,) = c.places(0, 10)[0][-1:], c.places(0, 10)[1][-1:]
    c.c.v_scales[0, p, 1, s, 0] = 255          # values 0 .. 31 of entry 9, KV head 1
    c.v[0][0][9, 1, :32] = np.nan
    (p,), (s,) = c.places(1, 5)[0][-1:], c.places(1, 5)[1][-1:]
    c.c.k_scales[0, p, 0, s, 1] = 255          # a key: every score with it
    c.k[0][1][4, 0, 32:] = np.nan
    case.run()
    got = case.out.double().cpu().numpy()
    assert np.isnan(got[:2, 2:, :32]).all() and not np.isnan(got[:2, 2:, 32:]).any() and not np.isnan(got[:2, :2]).any()
    assert np.isnan(got[2:, :2]).all() and not np.isnan(got[2:, 2:]).any()


def test_empty_rows_are_zero_and_have_no_weight():
    case = Case([0, 5, 0], [2, 1, 3], 4, 2, 64, 16, BF, "none").run()
    case.check()
    for r in (0, 1, 3, 4, 5):
        assert (case.out[r] == 0).all() and (case.lse[r] == -math.inf).all()
    before = case.cache.c.mass.clone()
    s2d2_kv4_weigh(case.cache.c, 0, case.rows)
    pages, slots = case.cache.places(1, 5)
    changed = (case.cache.c.mass != before).nonzero().cpu().numpy()
    assert {(int(p), int(s)) for _, p, _, s in changed} == {(int(p), int(s)) for p, s in zip(pages, slots)}


@pytest.mark.parametrize("scale", [1e-4, 3.0])
def test_flat_and_peaked_rows(scale):
    """Scores that hardly differ, and scores that differ by hundreds: the reference moves and stays."""
    for dtype in (BF, F32):
        case = Case([3000, 700], [2, 3], 4, 2, 64, 16, dtype, "causal", seed=5)
        case.scale = scale
        case.make()
        case.run().check()


def test_an_outlier_in_front_of_a_long_flat_cache():
    """One entry whose weight is 2^20 times the others': they keep theirs (together, a sixth of the row)."""
    n = 200000
    cache = P.Cache([n], 1, 32, 64, weights=False)
    k = np.zeros((n, 1, 32))
    k[0] = 6.0
    codes, scales = P.quantise(k)
    pages, slots = cache.places(0, n)
    at = torch.from_numpy(pages).to(DEV), torch.from_numpy(slots).to(DEV)
    cache.c.k_codes[0][at[0], :, at[1]] = torch.from_numpy(codes).to(DEV)
    cache.c.k_scales[0][at[0], :, at[1]] = torch.from_numpy(scales).to(DEV)
    cache.k[0][0] = P.values(codes, scales)
    q = torch.full((1, 1, 32), 1.0).to(BF).to(DEV)
    case = Case([n], [1], 1, 1, 32, 64, BF, "none", cache=cache)
    case.q = q
    case.scale = 20 * math.log(2) / (6 * 32)
    case.make()
    case.run().check()


def test_offsets_beyond_32_bits():
    cache = P.Cache([100, 33], 8, 128, 64, spare=0, pages_at=140000, weights=False)
    assert cache.c.k_codes.numel() > 1 << 32
    Case(cache.lens, [2, 1], 16, 8, 128, 64, BF, "causal", cache=cache).run().check()


def test_the_same_bits_again_on_another_stream_and_in_graphs_that_share_a_scratch():
    a = Case([5000, 300, 64], [4, 2, 7], 8, 2, 128, 16, BF, "block", seed=1)
    b = Case([5000, 2000, 10], [1, 40, 3], 8, 2, 128, 16, F32, "verify", seed=2)
    b.scratch = a.scratch = torch.full((max(a.scratch.numel(), b.scratch.numel()),), 255, dtype=torch.uint8, device=DEV)
    ref = []
    for c in (a, b):
        c.run().check()
        ref.append((c.out.clone(), c.lse.clone()))
        c.cache.c.mass.zero_()
        s2d2_kv4_weigh(c.cache.c, 0, c.rows)
        c.gained = c.cache.c.mass.clone()
    side = torch.cuda.Stream()
    for c, r in zip((a, b), ref):
        c.out.fill_(1)
        side.wait_stream(torch.cuda.current_stream())
        c.run(stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(c.out, r[0]) and torch.equal(c.lse, r[1])
    graphs = []
    for c in (a, b):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.run()
            s2d2_kv4_weigh(c.cache.c, 0, c.rows)
        graphs.append(g)
    for turn in range(3):
        for c, g, r in zip((a, b), graphs, ref):
            c.out.fill_(turn)
            c.lse.fill_(turn)
            c.cache.c.mass.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(c.out, r[0]) and torch.equal(c.lse, r[1]) and torch.equal(c.cache.c.mass, c.gained)


# ---- weigh ----

@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("hq,hkv,d,page,lens,counts", [(4, 2, 32, 16, [0, 1, 31, 32, 33, 300], [3, 1, 0, 6, 9, 40]), (7, 1, 64, 3, [100, 65], [5, 1]),
                                                       (16, 8, 128, 16, [2000, 40], [1, 33]), (10, 2, 256, 100, [64, 129], [7, 2])])
def test_weights_are_those_of_the_definition(dtype, hq, hkv, d, page, lens, counts):
    """Bound: a weight is off by its score's error, (d + 4) 2^-24 of the largest scale * sum |q||k|, and 2^-21; the lse it is given is off by half a step of
    its own, |lse| 2^-24; a sum of m weights of at most 1 in 32 bits by m 2^-24 of itself; the sum with the mass by 2^-24 of the result."""
    case = Case(lens, counts, hq, hkv, d, page, dtype, "causal", layers=2, layer=1, gap=1).run()
    lse = case.lse.clone()
    lse[case.row0[0]] = -math.inf       # a row without weight
    case.lse.copy_(lse)
    before = case.cache.c.mass.clone()
    s2d2_kv4_weigh(case.cache.c, 1, case.rows)
    got, seen = case.cache.c.mass.cpu(), torch.zeros(before.shape, dtype=torch.bool)
    want, most = P.weights(case.cache, 1, case.q.double().cpu().numpy(), case.row0, case.counts, case.scale, lse.double().cpu().numpy())
    rel = most * (d + 4) * 2.0 ** -24 + 2.0 ** -21 + 40 * 2.0 ** -24 + max(counts) * hq * 2.0 ** -24
    for i, s in enumerate(lens):
        pages, slots = (torch.from_numpy(t) for t in case.cache.places(i, s))
        old, new = before.cpu()[1][pages, :, slots].double().numpy(), got[1][pages, :, slots].double().numpy()
        assert (np.abs(new - old - want[i]) <= rel * want[i] + 2.0 ** -23 * (old + want[i])).all()
        if counts[i]:
            seen[1][pages, :, slots] = True
    assert torch.equal(got[~seen], before.cpu()[~seen])


def test_a_sequence_s_weights_add_up_to_its_rows():
    case = Case([700, 0, 45], [9, 3, 1], 8, 4, 128, 16, BF, "none").run()
    case.cache.c.mass.zero_()
    s2d2_kv4_weigh(case.cache.c, 0, case.rows)
    for i, s in enumerate(case.cache.lens):
        pages, slots = (torch.from_numpy(t).to(DEV) for t in case.cache.places(i, s))
        total = case.cache.c.mass[0][pages, :, slots].double().sum(0)
        if s:   # every row and head of the group gives 1
            assert (total - case.counts[i] * 2).abs().max() < case.counts[i] * 2 * 2.0 ** -16
