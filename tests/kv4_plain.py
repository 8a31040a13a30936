"""The operators on a 4-bit cache from their definitions, in 64 bits on the CPU, and caches for their tests."""
import math

import numpy as np
import torch

from paper_2603_25702_amd import Kv4Cache

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """codes [..., D / 2] and scale bytes [..., D / 32] of an array [..., D]; nearest level by search, ties to the even code."""
    x = np.asarray(x, np.float64)
    g = x.reshape(*x.shape[:-1], x.shape[-1] // 32, 32)
    fine = np.isfinite(g).all(-1)
    most = np.where(fine, np.abs(np.where(np.isfinite(g), g, 0)).max(-1), 0)
    e = np.full(most.shape, -23)
    for k in range(-23, 13):   # the smallest exponent that holds the largest value
        e = np.where(6 * 2.0 ** k < most, k + 1, e)
    y = np.where(fine[..., None], g, 0) / 2.0 ** e[..., None]
    off = np.abs(np.minimum(np.abs(y), 8)[..., None] - LEVELS)   # (cut: distances from 2^53 on would all be the same in 64 bits)
    even, odd = off[..., 0::2], off[..., 1::2]
    ke, ko = even.argmin(-1), odd.argmin(-1)
    code = np.where(even.min(-1) <= odd.min(-1), 2 * ke, 2 * ko + 1) + 8 * np.signbit(y)
    code = np.where(fine[..., None], code, 0).reshape(x.shape).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(fine, e + 127, 255).astype(np.uint8)


def values(codes, scales):
    codes, scales = np.asarray(codes), np.asarray(scales)
    c = np.stack((codes & 15, codes >> 4), -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    v = np.where(c & 8, -LEVELS[c & 7], LEVELS[c & 7])
    s = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return v * s.repeat(32, -1)


class Cache:
    """A cache with its contents on both sides: `c` on the device, k, v [layers, n][entries, Hkv, D] in 64 bits as the codes stand for."""

    def __init__(self, lens, hkv, d, page, layers=1, room=0, seed=0, weights=True, scale=1.0, spare=2, pages_at=0):
        rng = np.random.default_rng(seed)
        self.lens, self.hkv, self.d, self.page, self.layers = list(lens), hkv, d, page, layers
        n = len(lens)
        need = [-(-(s + room) // page) for s in lens]
        n_pages, wide = pages_at + sum(need) + spare, max(1, max(need))
        order = list(rng.permutation(np.arange(pages_at, n_pages)))
        self.table = np.full((n, wide), -1, np.int32)
        for i, k in enumerate(need):
            self.table[i, :k] = [order.pop() for _ in range(k)]
        dev = "cuda:0"
        shape = (layers, n_pages, hkv, page)
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
        noise = lambda last: torch.empty((*shape, last), dtype=torch.uint8, device=dev).random_(0, 256)  # noqa: E731
        # what no entry holds is noise: codes, and scales of which some read as NaN
        self.c = Kv4Cache(noise(d // 2), noise(d // 2), noise(d // 32).clamp_(min=130), noise(d // 32).clamp_(min=130), i32(self.table), i32(self.lens),
                          i32(self.lens), i32([0] * n), torch.rand(shape, device=dev) if weights else None,
                          torch.zeros(shape, dtype=torch.int32, device=dev) if weights else None)
        self.k, self.v = [], []
        for name, store in (("k", self.k), ("v", self.v)):
            for l in range(layers):
                per = []
                for i, s in enumerate(lens):
                    x = rng.standard_normal((s, hkv, d)) * scale * (np.where(rng.random((hkv, d)) < 0.05, 8, 1) if name == "k" else 1)
                    codes, scales = quantise(x)
                    per.append(values(codes, scales))
                    if s:
                        at = torch.from_numpy(self.table[i][np.arange(s) // page].astype(np.int64)), torch.from_numpy(np.arange(s) % page)
                        getattr(self.c, name + "_codes")[l][at[0], :, at[1]] = torch.from_numpy(codes).to(dev)
                        getattr(self.c, name + "_scales")[l][at[0], :, at[1]] = torch.from_numpy(scales).to(dev)
                store.append(per)

    def places(self, i, count):
        s = np.arange(count)
        return self.table[i][s // self.page].astype(np.int64), s % self.page

    def tensors(self):
        c = self.c
        return [t for t in (c.k_codes, c.v_codes, c.k_scales, c.v_scales, c.mass, c.position, c.entries, c.seq_len, c.status) if t is not None]


def attention(cache, layer, q, row0, counts, scale, k=None, v=None, lo=None, hi=None):
    """out [rows, Hq, D], lse [rows, Hq], and per output the sum of |weight * value| and per row the largest sum of |q||k| * scale (for error bounds)."""
    q = np.asarray(q, np.float64)
    rows, hq, d = q.shape
    out, lse = np.zeros((rows, hq, d)), np.full((rows, hq), -np.inf)
    absout, most = np.zeros((rows, hq, d)), np.zeros((rows, hq))
    grp = hq // cache.hkv
    with np.errstate(all="ignore"):
        for n, (r0, c) in enumerate(zip(row0, counts)):
            ck, cv = cache.k[layer][n], cache.v[layer][n]
            for r in range(r0, r0 + c):
                seen = []
                if k is not None:
                    a, b = (r0, r + 1) if lo is None else (lo[r], hi[r])
                    seen = [w for w in range(r0, r0 + c) if a <= w < b or w == r]
                for h in range(hq):
                    kk, vv = ck[:, h // grp], cv[:, h // grp]
                    if seen:
                        kk, vv = np.concatenate((kk, np.asarray(k, np.float64)[seen, h // grp])), np.concatenate((vv, np.asarray(v, np.float64)[seen, h // grp]))
                    if not len(kk):
                        continue
                    s = scale * (kk @ q[r, h])
                    m = s.max() if not np.isnan(s).any() else np.nan
                    p = np.exp(s - m)
                    lse[r, h] = m + np.log(p.sum())
                    p = p / p.sum()
                    out[r, h] = p @ vv
                    absout[r, h] = p @ np.abs(vv)
                    most[r, h] = scale * (np.abs(kk) @ np.abs(q[r, h])).max()
    return out, lse, absout, most


def weights(cache, layer, q, row0, counts, scale, lse):
    """[n][entries, Hkv]: what the rows give every entry; and its error bound's factor, the largest scale * sum |q||k|."""
    q, lse = np.asarray(q, np.float64), np.asarray(lse, np.float64)
    grp = q.shape[1] // cache.hkv
    out, most = [], 0.0
    for n, (r0, c) in enumerate(zip(row0, counts)):
        w = np.zeros((cache.lens[n], cache.hkv))
        for r in range(r0, r0 + c):
            for h in range(q.shape[1]):
                if lse[r, h] > -math.inf and cache.lens[n]:
                    w[:, h // grp] += np.exp(scale * (cache.k[layer][n][:, h // grp] @ q[r, h]) - lse[r, h])
                    most = max(most, scale * (np.abs(cache.k[layer][n][:, h // grp]) @ np.abs(q[r, h])).max())
        out.append(w)
    return out, most


def evict_list(mass, position, budget, sink, tail):
    """(places that are written, places they come from) of one list."""
    e = len(mass)
    safe = (position < sink) | (position >= tail)
    m = np.where(np.isnan(mass), -np.inf, mass.astype(np.float64))
    order = sorted(range(e), key=lambda i: (not safe[i], not np.isnan(mass[i]) and -m[i] or (np.inf if np.isnan(mass[i]) else 0.0), np.isnan(mass[i]) and not safe[i], i))
    keep = np.zeros(e, bool)
    keep[order[:budget]] = True
    s = np.arange(e)
    return s[:budget][~keep[:budget]], s[budget:][keep[budget:]]
