"""Quantising append and read of the 4-bit cache against the definition in 64 bits: bit for bit."""
import numpy as np
import pytest
import torch

from paper_2603_25702_amd import s2d2_kv4_append, s2d2_kv4_read

from . import kv4_plain as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def filled(cache, i, count, first=0):
    """(k codes, k scales, v codes, v scales, mass, position) of entries first .. of sequence i: [layers][count, ...]."""
    pages, slots = cache.places(i, first + count)
    at = torch.from_numpy(pages[first:]), torch.from_numpy(slots[first:])
    c = cache.c
    return [t.cpu()[:, at[0], :, at[1]].transpose(0, 1).numpy() for t in (c.k_codes, c.k_scales, c.v_codes, c.v_scales, c.mass, c.position)]


def every_group(dtype):
    """Groups whose largest value and whose others cover the type: all bf16 patterns in some group, ties between levels at several exponents, the borders
    where the exponent changes, subnormals, infinities and NaNs."""
    bits = np.arange(65536, dtype=np.uint32) << 16
    rows = [bits.view(np.float32).reshape(-1, 32)]                                     # neighbours: one exponent a group
    rng = np.random.default_rng(1)
    rows.append(rng.permutation(bits).view(np.float32).reshape(-1, 32))               # anything with anything: mostly NaN or saturated groups
    finite = bits.view(np.float32)[np.isfinite(bits.view(np.float32)) & (np.abs(bits.view(np.float32)) < 1e6)]
    rows.append(rng.permutation(finite)[: finite.size // 32 * 32].reshape(-1, 32))
    grid = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 5.96875], np.float32)
    near = np.concatenate((grid, np.nextafter(grid, np.float32(9), dtype=np.float32))) if dtype == torch.float32 else np.concatenate((grid, -grid))
    rows += [np.float32(2.0 ** e) * near[None] for e in range(-30, 16)]
    rows += [np.float32(m) * np.ones((1, 32), np.float32) for m in (6.0, 6.0000005, 5.9999995, 49152, 49153, 60000, 3e38, 1e-40, 2 ** -24, 2 ** -25, -6.03125)]
    rows.append((rng.standard_normal((4096, 32)) * 10.0 ** rng.uniform(-7, 5, (4096, 1))).astype(np.float32))
    return np.concatenate(rows)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("hkv,d", [(3, 64), (1, 32), (2, 128), (5, 256)])
def test_codes_and_scales_are_those_of_the_definition(dtype, hkv, d):
    groups = every_group(dtype)
    per_row = hkv * d // 32
    total = len(groups) // per_row
    x = torch.from_numpy(groups[: total * per_row].reshape(total, hkv, d)).to(dtype)
    cache = P.Cache([0], hkv, d, 16, room=total)
    k, v = x[None].to(DEV), x.flip(0)[None].to(DEV)
    s2d2_kv4_append(cache.c, k, v, i32([0]), i32([total]), total)
    kc, ks, vc, vs, mass, position = (t[0] for t in filled(cache, 0, total))
    for got_c, got_s, want in ((kc, ks, x), (vc, vs, x.flip(0))):
        codes, scales = P.quantise(want.double().numpy())
        assert np.array_equal(got_s, scales)
        assert np.array_equal(got_c, codes)
    assert (mass == 0).all() and np.array_equal(position, np.broadcast_to(np.arange(total)[:, None], position.shape))
    for back_type in (torch.bfloat16, torch.float32):
        kb, vb = (torch.empty(1, 1, total, hkv, d, dtype=back_type, device=DEV) for _ in range(2))
        s2d2_kv4_read(cache.c, i32([0]), kb, vb)
        assert np.array_equal(kb[0, 0].double().cpu().numpy(), P.values(kc, ks), equal_nan=True)
        assert np.array_equal(vb[0, 0].double().cpu().numpy(), P.values(vc, vs), equal_nan=True)


@pytest.mark.parametrize("page", [1, 3, 16, 100])
@pytest.mark.parametrize("dtype,hkv,d,layers", [(torch.bfloat16, 8, 128, 3), (torch.float32, 1, 32, 1), (torch.bfloat16, 5, 256, 2), (torch.float32, 2, 64, 4)])
def test_ragged_rows_go_behind_the_entries_and_nowhere_else(page, dtype, hkv, d, layers):
    lens, counts = [0, 1, 33, 100, 7, 60], [5, 0, 17, 4, 1, 9]
    T = 17
    cache = P.Cache(lens, hkv, d, page, layers=layers, room=T, seed=page)
    cache.c.seq_len += 1000     # (positions go by seq_len, places by entries)
    gen = torch.Generator().manual_seed(page)
    row0 = np.array([0, 0, 6, 30, 40, 41])      # rows that no sequence has lie between
    wide = torch.randn(layers, 60, hkv + 1, d, generator=gen).to(dtype).to(DEV)
    k, v = wide[:, :, 1:], torch.randn(layers, 60, hkv + 1, d, generator=gen).to(dtype).to(DEV)[:, :, 1:]   # rows further apart than they are long
    before = [t.clone() for t in cache.tensors()]
    want = [t.clone() for t in before]
    s2d2_kv4_append(cache.c, k, v, i32(row0), i32(counts), T)
    pos0 = before[-2].cpu().numpy()
    for i, c in enumerate(counts):
        if not c:
            continue
        pages, slots = cache.places(i, lens[i] + c)
        at = torch.from_numpy(pages[lens[i]:]).to(DEV), torch.from_numpy(slots[lens[i]:]).to(DEV)
        for l in range(layers):
            for src, cd, sc in ((k, want[0], want[2]), (v, want[1], want[3])):
                codes, scales = P.quantise(src[l, row0[i]:row0[i] + c].double().cpu().numpy())
                cd[l][at[0], :, at[1]] = torch.from_numpy(codes).to(DEV)
                sc[l][at[0], :, at[1]] = torch.from_numpy(scales).to(DEV)
            want[4][l][at[0], :, at[1]] = 0.0
            want[5][l][at[0], :, at[1]] = i32(pos0[i] + np.arange(c))[:, None].expand(c, hkv)
    want[6] += i32(counts)
    want[7] += i32(counts)
    for got, w in zip(cache.tensors(), want):
        assert torch.equal(got, w)
    # all entries back, old and new, from a place of each sequence's own; what lies behind is left as it was
    first = np.array([0, 0, 20, 101, 3, -2])
    kb, vb = (torch.full((layers, 6, 40, hkv, d), 77.0, dtype=dtype, device=DEV) for _ in range(2))
    s2d2_kv4_read(cache.c, i32(first), kb, vb)
    for i in range(6):
        for t in range(40):
            e = first[i] + t
            if 0 <= e < lens[i] + counts[i]:
                (p,), (s,) = cache.table[i][[e // page]], [e % page]
                for back, cd, sc in ((kb, want[0], want[2]), (vb, want[1], want[3])):
                    if t % 7 == 0:
                        assert np.array_equal(back[:, i, t].double().cpu().numpy(), P.values(cd[:, p, :, s].cpu().numpy(), sc[:, p, :, s].cpu().numpy()))
            else:
                assert (kb[:, i, t] == 77).all() and (vb[:, i, t] == 77).all()


def test_counts_out_of_range_no_room_and_pages_that_are_not_there():
    hkv, d, page, T = 2, 64, 4, 6
    lens = [3, 4, 8, 2, 5, 6]
    cache = P.Cache(lens, hkv, d, page, room=8)
    cap = cache.table.shape[1] * page
    counts = [-5, 100, 6, 6, 6, 6]              # below zero, above T (cut to 6), as they are
    row0 = [0, 0, 35, -1, 6, 12]                # the third and the fourth sequence's rows leave the tensor
    cache.table[4, 2] = -7                      # a page outside the cache: its entries are not written
    cache.c.page_table.copy_(torch.from_numpy(cache.table))
    cache.c.entries[5] = cap - 5                # room for five
    lens[5] = cap - 5
    x = torch.randn(1, 40, hkv, d, device=DEV)
    before = [t.clone() for t in cache.tensors()]
    s2d2_kv4_append(cache.c, x, x, i32(row0), i32(counts), T)
    after = cache.tensors()
    assert after[6].tolist() == [3, 10, 8, 2, 11, cap - 5]
    assert after[7].tolist() == [3, 10, 8, 2, 11, 6]
    assert after[8].tolist() == [0, 0, 0, 0, 0, -2]
    written = torch.zeros(cache.c.mass.shape, dtype=torch.bool)
    for i in (1, 4):
        pages, slots = cache.places(i, lens[i] + 6)
        for p, s in list(zip(pages, slots))[lens[i]:]:
            if p >= 0:
                written[0, p, :, s] = True
    for a, b in zip(after[:6], before[:6]):
        same = (a == b).cpu()
        same = same if same.dim() == 4 else same.flatten(4).all(-1)
        assert same[~written].all()
    assert (after[4].cpu()[written] == 0).all()


def test_a_cache_without_mass_and_position_and_without_status():
    cache = P.Cache([2, 0], 1, 32, 8, room=8, weights=False)
    cache.c._view.status = None
    x = torch.randn(1, 8, 1, 32, device=DEV)
    s2d2_kv4_append(cache.c, x, x, i32([0, 3]), i32([3, 5]), 5)
    assert cache.c.entries.tolist() == [5, 5]
    cache.c.entries[0] = 15
    s2d2_kv4_append(cache.c, x, x, i32([0, 3]), i32([3, 0]), 5)
    assert cache.c.entries.tolist() == [15, 5]


def test_offsets_beyond_32_bits():
    """Codes of more than 4 GiB: the entries lie in the last pages, one layer behind 2^32 bytes."""
    hkv, d, page = 8, 128, 64
    cache = P.Cache([100, 3], hkv, d, page, layers=1, room=64, spare=0, pages_at=140000, weights=False)
    assert cache.c.k_codes.numel() > 1 << 32
    x = torch.randn(1, 20, hkv, d, device=DEV).bfloat16()
    s2d2_kv4_append(cache.c, x, x * 2, i32([0, 12]), i32([12, 8]), 12)
    kb, vb = (torch.empty(1, 2, 12, hkv, d, device=DEV) for _ in range(2))
    s2d2_kv4_read(cache.c, i32([100, 3]), kb, vb)
    for back, src in ((kb, x), (vb, x * 2)):
        want = P.values(*P.quantise(src[0].double().cpu().numpy()))
        assert np.array_equal(back[0, 0].double().cpu().numpy(), want[:12]) and np.array_equal(back[0, 1, :8].double().cpu().numpy(), want[12:])
    s2d2_kv4_read(cache.c, i32([88, 0]), kb, vb)
    assert np.array_equal(kb[0, 0].double().cpu().numpy(), cache.k[0][0][88:100]) and np.array_equal(vb[0, 1, :3].double().cpu().numpy(), cache.v[0][1])
