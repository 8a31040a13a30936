"""Refusals of the 4-bit cache's calls at the ends of the types, on the CPU."""
import pytest

from paper_2603_25702_amd import binding as Bd

from .test_kv4_abi import FAKE, lib, rows, view  # noqa: F401


@pytest.mark.parametrize("scale,refused", [(2.3e38, False), (2.4e38, True), (3.4e38, True)])
def test_scales_whose_product_with_log2_e_overflows_are_refused(lib, scale, refused):  # noqa: F811
    """Scores are taken to base 2: scale * 1.4427 has to be finite.  (A scratch that is too small ends the calls that are not refused.)"""
    big = view(max_pages_per_seq=1024)
    assert lib.s2d2_kv4_attention(None, big, 0, rows(scale=scale), FAKE, 16) == (Bd.S2D2_EINVAL if refused else Bd.S2D2_ENOSPC)
    if refused:
        assert lib.s2d2_kv4_weigh(None, view(), 0, rows(scale=scale)) == Bd.S2D2_EINVAL
