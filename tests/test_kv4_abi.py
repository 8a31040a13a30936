"""Host-side checks of the 4-bit cache's C entry points that need no GPU: exports, struct layout, refusals before anything is launched."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

from paper_2603_25702_amd import binding as Bd
from paper_2603_25702_amd import build, kv4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, EINVAL, ENOSPC = Bd.S2D2_OK, Bd.S2D2_EINVAL, Bd.S2D2_ENOSPC
FAKE = 0x7F0000000000


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(Bd.lib_path()):
        build.build_lib()
    return kv4._lib()


def view(**kw):
    w = kv4.Kv4View(*[FAKE] * 10, 2, 64, 16, 32, 8, 128)
    for k, v in kw.items():
        setattr(w, k, v)
    return w


def rows(**kw):
    r = kv4.Kv4RowsC(4, 8, 32, 32, Bd.S2D2_BF16, 0.1, FAKE, FAKE, FAKE, 32 * 128, 8 * 128, 32 * 128, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE)
    for k, v in kw.items():
        setattr(r, k, v)
    return r


def test_every_declared_symbol_is_exported(lib):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "s2d2_kv4.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(s2d2_[a-z_0-9]+)\s*\(", text))
    assert names == set(kv4.EXPORTS)
    for n in names:
        assert getattr(lib, n) is not None
    driver = open(os.path.join(ROOT, "tests", "host", "kv4_check.cpp")).read()
    assert [n for n in names if n + "(" not in driver] == []


def test_struct_sizes_match_the_header_layout():
    assert C.sizeof(kv4.Kv4View) == 10 * 8 + 6 * 4
    assert C.sizeof(kv4.Kv4RowsC) == 6 * 4 + 3 * 8 + 3 * 8 + 6 * 8


BAD_VIEWS = [("k_codes", 0), ("v_codes", None), ("k_scales", None), ("v_scales", FAKE + 4), ("k_codes", FAKE + 8), ("mass", FAKE + 2), ("position", FAKE + 1),
             ("page_table", None), ("entries", None), ("seq_len", None), ("n_layers", 0), ("n_pages", 0), ("page_size", 0), ("page_size", 1 << 26),
             ("max_pages_per_seq", -1), ("n_kv_heads", 0), ("n_kv_heads", 1025), ("head_dim", 96), ("head_dim", 0)]


@pytest.mark.parametrize("field,value", BAD_VIEWS)
def test_bad_caches_are_refused_by_every_call(lib, field, value):
    w = view(**{field: value})
    assert lib.s2d2_kv4_append(None, w, 4, 8, 32, 1, FAKE, FAKE, 1 << 20, 1024, FAKE, FAKE) == EINVAL
    assert lib.s2d2_kv4_read(None, w, 4, 8, 1, FAKE, FAKE, FAKE) == EINVAL
    assert lib.s2d2_kv4_attention_bytes(w, 4, 8, 32) == EINVAL
    assert lib.s2d2_kv4_attention(None, w, 0, rows(), FAKE, 1 << 40) == EINVAL
    assert lib.s2d2_kv4_weigh(None, w, 0, rows()) == EINVAL
    assert lib.s2d2_kv4_evict(None, w, 4, 100, 0, 0, 0, FAKE, 1 << 40) == EINVAL
    assert lib.s2d2_kv4_evict_bytes(w, 4) == EINVAL
    assert b"4-bit cache" in lib.s2d2_last_error()


BAD_ROWS = [("N", 0), ("N", 1025), ("T", 0), ("T", 8193), ("rows", 0), ("n_q_heads", 12), ("n_q_heads", 0), ("n_q_heads", 2048), ("dtype", 2), ("scale", 0.0),
            ("scale", -1.0), ("scale", float("nan")), ("scale", float("inf")), ("q", None), ("q", FAKE + 2), ("q_stride", 32 * 128 - 8), ("q_stride", 32 * 128 + 4),
            ("q_stride", 1 << 40), ("row0", None), ("n_rows", None), ("n_rows", FAKE + 1), ("lo", FAKE + 2)]


@pytest.mark.parametrize("field,value", BAD_ROWS)
def test_bad_rows_are_refused(lib, field, value):
    assert lib.s2d2_kv4_attention(None, view(), 0, rows(**{field: value}), FAKE, 1 << 40) == EINVAL
    assert lib.s2d2_kv4_weigh(None, view(), 0, rows(**{field: value})) == EINVAL


@pytest.mark.parametrize("field,value", [("k", None), ("v", None), ("k", FAKE + 4), ("kv_stride", 8 * 128 - 8), ("kv_stride", 8 * 128 + 2), ("lo", None), ("hi", None),
                                         ("out", None), ("out", FAKE + 8), ("out_stride", 0)])
def test_bad_windows_and_outputs_are_refused(lib, field, value):
    assert lib.s2d2_kv4_attention(None, view(), 0, rows(**{field: value}), FAKE, 1 << 40) == EINVAL


def test_other_refusals(lib):
    w = view()
    for layer in (-1, 2):
        assert lib.s2d2_kv4_attention(None, w, layer, rows(), FAKE, 1 << 40) == EINVAL
        assert lib.s2d2_kv4_weigh(None, w, layer, rows()) == EINVAL
    assert lib.s2d2_kv4_attention(None, w, 0, None, FAKE, 1 << 40) == EINVAL
    huge = view(max_pages_per_seq=(1 << 26) - 1)
    assert lib.s2d2_kv4_attention_bytes(huge, 63, 8, 32) > 0 and lib.s2d2_kv4_attention_bytes(huge, 64, 8, 32) == EINVAL   # 64 * (2^30 - 16 + 8 + 64) >= 2^36
    assert lib.s2d2_kv4_weigh(None, huge, 0, rows(N=100)) == EINVAL and lib.s2d2_kv4_attention(None, huge, 0, rows(N=100), FAKE, 1 << 60) == EINVAL
    assert lib.s2d2_kv4_attention_bytes(w, 128, 8192, 32) > 0 and lib.s2d2_kv4_attention_bytes(w, 129, 8192, 32) == EINVAL
    assert lib.s2d2_kv4_evict_bytes(view(n_layers=4096, n_kv_heads=1024), 1) == EINVAL
    assert lib.s2d2_kv4_append(None, w, 1024, 1 << 16, 32, 1, FAKE, FAKE, 1 << 20, 1024, FAKE, FAKE) == EINVAL
    assert lib.s2d2_kv4_read(None, w, 1024, 1 << 16, 1, FAKE, FAKE, FAKE) == EINVAL
    big = view(max_pages_per_seq=1024)
    need = lib.s2d2_kv4_attention_bytes(big, 4, 8, 32)
    assert need > 0
    assert lib.s2d2_kv4_attention(None, big, 0, rows(), FAKE, need - 1) == ENOSPC
    assert lib.s2d2_kv4_attention(None, big, 0, rows(), FAKE + 8, need) == EINVAL
    assert lib.s2d2_kv4_attention(None, big, 0, rows(), None, need) == EINVAL
    assert lib.s2d2_kv4_weigh(None, w, 0, rows(lse=None)) == EINVAL
    assert lib.s2d2_kv4_weigh(None, view(mass=None), 0, rows()) == EINVAL
    for n, budget, slack, sink, recent in ((0, 8, 0, 0, 0), (1025, 8, 0, 0, 0), (4, 0, 0, 0, 0), (4, 8, -1, 0, 0), (4, 8, 0, -1, 0), (4, 8, 0, 0, -1), (4, 8, 0, 5, 4),
                                           (4, 8, 0, 2**31 - 1, 2**31 - 1)):
        assert lib.s2d2_kv4_evict(None, w, n, budget, slack, sink, recent, FAKE, 1 << 40) == EINVAL
    assert lib.s2d2_kv4_evict(None, view(mass=None), 4, 8, 0, 0, 0, FAKE, 1 << 40) == EINVAL
    assert lib.s2d2_kv4_evict(None, view(position=None), 4, 8, 0, 0, 0, FAKE, 1 << 40) == EINVAL
    need = lib.s2d2_kv4_evict_bytes(w, 4)
    assert need >= 4 * 2 * 4 * 8 * (1 + 32 * 16) and lib.s2d2_kv4_evict_bytes(w, 0) == EINVAL
    assert lib.s2d2_kv4_evict(None, w, 4, 8, 0, 0, 0, FAKE, need - 1) == ENOSPC
    assert lib.s2d2_kv4_evict(None, w, 4, 8, 0, 0, 0, FAKE + 2, need) == EINVAL
    assert lib.s2d2_kv4_evict(None, w, 4, 8, 0, 0, 0, None, need) == EINVAL
    good = (w, 4, 8, 32, 1, FAKE, FAKE, 1 << 20, 1024, FAKE, FAKE)
    for at, bad in ((1, 0), (1, 1025), (2, 0), (3, 0), (4, 7), (5, None), (5, FAKE + 8), (6, None), (7, 512), (7, 1025 * 1024 + 4), (7, -1024), (8, 1016), (8, 1028), (9, None), (10, FAKE + 2)):
        assert lib.s2d2_kv4_append(None, *good[:at], bad, *good[at + 1:]) == EINVAL, at
    good = (w, 4, 8, 1, FAKE, FAKE, FAKE)
    for at, bad in ((1, 0), (2, 0), (3, 5), (4, None), (5, None), (6, FAKE + 4)):
        assert lib.s2d2_kv4_read(None, *good[:at], bad, *good[at + 1:]) == EINVAL, at
    assert lib.s2d2_set_kv4(None, w, FAKE, 1 << 40, FAKE) == EINVAL


def test_scratch_grows_with_the_batch_and_never_with_a_smaller_one(lib):
    for cap, hkv, hq, d in ((512, 8, 32, 128), (64, 1, 7, 64), (4096, 5, 35, 256), (1 << 16, 4, 16, 32)):
        w = view(max_pages_per_seq=cap, n_kv_heads=hkv, head_dim=d)
        for n in (1, 3, 16, 1024):
            last = 0
            for t in (1, 2, 5, 8, 9, 31, 32, 64, 192, 1000, 8192):
                if n * t * hq > 1 << 25:
                    break
                b = lib.s2d2_kv4_attention_bytes(w, n, t, hq)
                assert b >= last and b >= lib.s2d2_kv4_attention_bytes(w, max(1, n // 2), t, hq)
                last = b


def test_the_binding_refuses_tensors_that_do_not_fit():
    with pytest.raises(Bd.S2D2Error, match="GPU"):
        kv4.Kv4Cache(torch.zeros(1, 2, 1, 4, 16, dtype=torch.uint8), *[None] * 6)
    with pytest.raises(Bd.S2D2Error, match="k_codes"):
        kv4.Kv4Cache(torch.zeros(1, 2, 1, 4, 16), *[None] * 6)
    q, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
    kv4.Kv4Rows(q, i, i, 4, 0.1, out=torch.zeros_like(q))
    for bad in (dict(q=q.half()), dict(q=q[0]), dict(out=torch.zeros(4, 2, 64)), dict(out=torch.zeros(4, 64, 2, dtype=torch.bfloat16).transpose(1, 2)), dict(row0=i.long()),
                dict(n_rows=torch.zeros(2, dtype=torch.int32)), dict(k=q), dict(lo=torch.zeros(4, dtype=torch.int32)), dict(lse=torch.zeros(4, 3)),
                dict(k=q, v=torch.zeros(4, 4, 64, dtype=torch.bfloat16)[:, :2])):
        with pytest.raises(Bd.S2D2Error):
            kv4.Kv4Rows(**{**dict(q=q, row0=i, n_rows=i, T=4, scale=0.1), **bad})


def test_argument_checks_and_size_arithmetic_are_clean_under_asan_and_ubsan():
    exe = build.build_host_check("kv4_check")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    env.pop("LD_PRELOAD", None)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-3000:]
    assert "kv4_check: 0 failed expectation(s)" in r.stdout
