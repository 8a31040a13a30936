"""fp32 rows on the 4-bit cache keep the bits of fp32: weights far below the largest, finite values up to the type's largest; and rows beside those that are NaN.

Error bound of fp32 rows, relative to sum p |v|: a score is a sum of D products in 32 bits, off by at most D * 2^-24 * sum |q||k| times scale; scaling and exponent
add 4 * 2^-24 of the same magnitude and 2^-21; weights relative to their sum are off by twice that.  Weights are split into three planes of bf16: 2^-24 of each, whatever its size.  Sums of n terms: sqrt(n) * 2^-24 * 8; the output 2^-21.
What 32 bits cannot hold: an exponential below 2^-126 is 0, and so is a plane of one.  The largest weight of a row is at least 2^7 by the choice of the reference, and the three planes of a
weight lose less than 3 * 2^-126: per key less than 2^-131 of the row's sum, times its |v|."""
import math

import numpy as np
import pytest
import torch

from . import kv4_plain as P
from .test_gpu_kv4_attention import BF, DEV, F32, Case

pytestmark = pytest.mark.gpu


def check_fp32(case):
    """Without a term for small weights: each is as exact, relative to itself, as the largest."""
    out, lse, absout, most = case.want()
    d, n = out.shape[2], max(case.cache.lens + [1]) + case.T
    rel = 2 * (most[..., None] * (d + 4) * 2.0 ** -24 + 2.0 ** -21) + 8 * math.sqrt(n) * 2.0 ** -24 + 2.0 ** -21
    off = np.abs(case.out.double().cpu().numpy() - out)
    vmost = max([np.abs(x).max() for x in case.cache.v[case.layer] if x.size] + ([case.v.abs().max().item()] if case.v is not None else []))
    room = rel * absout + n * 2.0 ** -131 * vmost
    assert bool((off <= room).all()), f"worst {np.nanmax(off / room):.2f} of the bound"


def write(cache, name, values):
    """All entries of a cache of one sequence."""
    codes, scales = P.quantise(values)
    pages, slots = cache.places(0, len(values))
    at = torch.from_numpy(pages).to(DEV), torch.from_numpy(slots).to(DEV)
    getattr(cache.c, name + "_codes")[0][at[0], :, at[1]] = torch.from_numpy(codes).to(DEV)
    getattr(cache.c, name + "_scales")[0][at[0], :, at[1]] = torch.from_numpy(scales).to(DEV)
    getattr(cache, name)[0][0] = P.values(codes, scales)


@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("bits", [12.3, 20.7, 40.1])
def test_weights_far_below_the_largest_keep_their_bits(d, bits):
    """Entry 0 outweighs each of the others by 2^bits and has the value 0: the output is what the others give."""
    for n in (32, 200):
        cache = P.Cache([n], 1, d, 16, weights=False, seed=n)
        k, v = np.zeros((n, 1, d)), np.random.default_rng(n).standard_normal((n, 1, d))
        k[0], v[0] = 6.0, 0.0
        write(cache, "k", k)
        write(cache, "v", v)
        case = Case([n], [1], 1, 1, d, 16, F32, "none", cache=cache)
        case.q.fill_(1.0)
        case.scale = bits * math.log(2) / (6 * d)
        case.make()
        check_fp32(case.run())


@pytest.mark.parametrize("hq,hkv,d,page", [(4, 2, 32, 16), (7, 1, 64, 3), (8, 8, 128, 16), (4, 2, 256, 100)])
@pytest.mark.parametrize("scale", [1e-3, 0.2, 2.0])
def test_fp32_rows_of_flat_and_peaked_weights(hq, hkv, d, page, scale):
    case = Case([300, 33, 1], [3, 9, 2], hq, hkv, d, page, F32, "causal", seed=d)
    case.scale = scale
    case.make()
    check_fp32(case.run())


def test_finite_values_up_to_the_largest():
    """Window rows of fp32 beyond bf16's largest value, 3.39e38, and queries against small keys; values of up to 2^100 of rows that are seen in full."""
    big = 3.4e38
    case = Case([40], [4], 2, 2, 64, 16, F32, "causal", seed=8)
    case.k[1, 0, 5] = big           # rows 1, 2, 3 see it: 8 of their scores
    case.q[:, 0, 5] = 2.0 ** -125
    case.make()
    check_fp32(case.run())
    case = Case([40], [4], 2, 2, 64, 16, F32, "causal", seed=9)
    case.q[2, 1, 7] = -big          # against keys that are 0 there
    case.k[:, 1, 7] = 0
    c = case.cache
    c.k[0][0][:, 1, :32] = 0
    pages, slots = c.places(0, 40)
    c.c.k_codes[0, torch.from_numpy(pages), 1, torch.from_numpy(slots), :16] = 0
    case.make()
    check_fp32(case.run())
    for dtype in (BF, F32):
        case = Case([40], [4], 2, 2, 64, 16, dtype, "causal", seed=10)
        case.v.mul_(2.0 ** 98)
        case.make()
        case.run().check()


def test_a_finite_value_above_bf16_s_largest_is_no_infinity():
    case = Case([0], [3], 1, 1, 32, 16, F32, "causal", seed=11)
    case.q.fill_(1.0)
    case.k.fill_(0.0)
    case.k[1] = -3.0                # its weight in rows 1 and 2 against row 0's: exp(-96 * scale)
    case.scale = 0.5
    case.v.fill_(1.0)
    case.v[1] = 3.4e38
    case.k[2] = -100.0
    case.make()
    case.run()
    out, lse, absout, most = case.want()
    got = case.out.double().cpu().numpy()
    assert np.isfinite(got).all()
    rel = 2 * (most[..., None] * 36 * 2.0 ** -24 + 2.0 ** -21) + 2.0 ** -20
    assert (np.abs(got - out) <= rel * absout).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_heads_and_rows_beside_a_value_that_is_not_finite(dtype, what):
    """One value of one KV head of a window row: the heads of that KV head in the rows that see it are NaN, all others are right."""
    case = Case([40, 0, 70], [6, 6, 6], 6, 3, 64, 16, dtype, "verify", gap=2, seed=12)
    at = [case.row0[0] + 5, case.row0[1] + 1, case.row0[2] + 2]
    for r in at:
        case.v[r, 1, 3] = what
    case.make()
    case.run()
    with np.errstate(all="ignore"):
        out, lse, absout, most = case.want()
    for r0, bad in zip(case.row0, at):
        for t in range(6):
            sees = r0 + t == bad or case.lo[r0 + t] <= bad < case.hi[r0 + t]
            got = torch.isnan(case.out[r0 + t]).all(-1).tolist()
            assert got == [sees and h // 2 == 1 for h in range(6)], (r0, t)
            for store in (out, absout, case.out):
                if sees:
                    store[r0 + t, 2:4] = math.nan
            if sees:
                lse[r0 + t, 2:4] = math.nan
                case.lse[r0 + t, 2:4] = math.nan
    case.check((out, lse, absout, most))
