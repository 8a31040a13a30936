"""Eviction from the 4-bit cache against its definition: the whole cache, bit for bit."""
import math

import numpy as np
import pytest
import torch

from paper_2603_25702_amd import s2d2_kv4_evict

from . import kv4_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def prepared(lens, hkv=2, d=64, page=16, layers=2, seed=0, mass=None, spread=1.0):
    cache = P.Cache(lens, hkv, d, page, layers=layers, seed=seed)
    rng = np.random.default_rng(seed)
    for i, s in enumerate(lens):
        pages, slots = (torch.from_numpy(t).to(DEV) for t in cache.places(i, s))
        m = mass(rng, (s, layers, hkv)) if mass else rng.exponential(1.0, (s, layers, hkv)) * spread
        cache.c.mass[:, pages, :, slots] = torch.from_numpy(m.astype(np.float32)).to(DEV)
        # positions in any order, with gaps: 3 * a permutation
        p = np.stack([np.stack([rng.permutation(s) * 3 for _ in range(hkv)], -1) for _ in range(layers)], 1) if s else np.zeros((0, layers, hkv))
        cache.c.position[:, pages, :, slots] = torch.from_numpy(p.astype(np.int32)).to(DEV)
    cache.c.seq_len.copy_(torch.tensor([3 * s for s in lens]))
    return cache


def expected(cache, budget, slack, sink, recent):
    """The cache's tensors after the definition's moves, and how many there were."""
    want = [t.cpu().clone() for t in cache.tensors()]
    moved = 0
    for i in range(len(cache.lens)):
        e = max(0, min(int(want[6][i]), cache.table.shape[1] * cache.page))
        if e <= budget + slack:
            continue
        pages, slots = cache.places(i, e)
        for l in range(cache.layers):
            for h in range(cache.hkv):
                to, source = P.evict_list(want[4][l, pages, h, slots].numpy(), want[5][l, pages, h, slots].numpy(), budget, sink, int(want[7][i]) - recent)
                assert len(to) == len(source)
                moved += len(to)
                for t in want[:6]:
                    t[l, pages[to], h, slots[to]] = t[l, pages[source], h, slots[source]]
        want[6][i] = budget
    return want, moved


def check(cache, budget, slack=0, sink=0, recent=0, moves=True):
    want, moved = expected(cache, budget, slack, sink, recent)
    assert (moved > 0) == moves
    s2d2_kv4_evict(cache.c, budget, slack, sink, recent)
    for name, got, w in zip("k_codes v_codes k_scales v_scales mass position entries seq_len status".split(), cache.tensors(), want):
        assert torch.equal(got.cpu().view(torch.int32) if got.dtype == torch.float32 else got.cpu(), w.view(torch.int32) if w.dtype == torch.float32 else w), name


@pytest.mark.parametrize("hkv,d,page", [(2, 64, 16), (1, 32, 3), (3, 128, 100), (2, 256, 1)])
@pytest.mark.parametrize("budget,sink,recent", [(1, 0, 0), (40, 4, 16), (64, 0, 64), (65, 10, 0), (200, 7, 90)])
def test_lists_of_all_lengths(hkv, d, page, budget, sink, recent):
    check(prepared([0, 1, 2, 40, 41, 64, 65, 66, 201, 333], hkv, d, page, seed=budget), budget, 0, sink, recent)


def test_budget_and_slack():
    lens = [100, 110, 111, 120]
    check(prepared(lens), 100, 10)                     # 111 and 120 are cut, 110 is not
    cache = prepared(lens)
    check(cache, 100, 20, moves=False)
    check(cache, 2 ** 31 - 1, 2 ** 31 - 1, moves=False)
    check(cache, 100, 2 ** 31 - 1, moves=False)
    check(cache, 1, 0)
    check(cache, 1, 0, moves=False)                    # nothing left to do


@pytest.mark.parametrize("mass", [lambda r, s: np.zeros(s), lambda r, s: np.full(s, 0.25), lambda r, s: r.integers(0, 3, s) * 1.0,
                                  lambda r, s: np.where(r.random(s) < 0.5, -0.0, 0.0), lambda r, s: np.where(r.random(s) < 0.3, math.nan, r.random(s)),
                                  lambda r, s: np.where(r.random(s) < 0.3, math.inf, r.integers(0, 2, s)), lambda r, s: -r.random(s) + 0.3,
                                  lambda r, s: 1.0 + r.integers(0, 5, s) * 2.0 ** -23, lambda r, s: r.random(s) * 1e-42])
def test_ties_and_masses_of_every_kind(mass):
    check(prepared([300, 77, 1200], mass=mass, seed=3), 70, 0, 5, 9)


def test_all_of_the_budget_is_protected():
    check(prepared([500]), 30, 0, 30, 0)
    check(prepared([500]), 30, 0, 12, 18)


@pytest.mark.parametrize("entries,budget", [(4160, 4096), (32768, 4096), (33000, 32000), (40000, 100), (70000, 35000)])
def test_long_lists(entries, budget):
    """Lists whose keys do not fit into LDS, and more moves than are listed at a time."""
    check(prepared([entries, 50], hkv=1, d=32, page=64, layers=1), budget, 0, 4, 32)


def test_table_entries_that_are_no_pages():
    """An entry in a page outside the cache is read as in the nearest page and never written."""
    cache = prepared([64], hkv=1, layers=1, page=16)
    cache.table[0, 1] = 10 ** 6
    cache.c.page_table.copy_(torch.from_numpy(cache.table))
    before = [t.clone() for t in cache.tensors()]
    s2d2_kv4_evict(cache.c, 32)
    assert cache.c.entries.tolist() == [32]
    mine = torch.zeros(cache.c.n_pages, dtype=torch.bool)
    mine[int(cache.table[0, 0])] = True
    for a, b in zip(cache.tensors()[:6], before[:6]):
        assert torch.equal(a.cpu()[:, ~mine], b.cpu()[:, ~mine])


def test_the_same_bits_in_a_graph_on_every_replay():
    cache = prepared([900, 300, 20], hkv=4, d=128)
    start = [t.clone() for t in cache.tensors()]
    s2d2_kv4_evict(cache.c, 128, 16, 4, 32)
    want = [t.clone() for t in cache.tensors()]
    for t, s in zip(cache.tensors(), start):
        t.copy_(s)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s2d2_kv4_evict(cache.c, 128, 16, 4, 32)
    for _ in range(3):
        for t, s in zip(cache.tensors(), start):
            t.copy_(s)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(cache.tensors(), want))
