"""Sizes and values at the ends of what the attention calls take, refused or not before any launch (host only)."""
import ctypes

import pytest

from paper_2606_08635_amd import skv

P = 4096  # an aligned address that no refused call dereferences


def _size(B, Lq, Hq, H=1, d=32, max_len=0, prefix=0):
    cfg = skv._DECODE_CONFIG.pack(0, B, Lq, Hq, H, d, 1, 1, 0, max_len, prefix, 0, 1.0, *[0] * 9)
    out = ctypes.c_uint64()
    return skv.lib().skv_attn_decode_workspace_size(cfg, ctypes.byref(out))


def _decode(B, Lq, Hq, H=1, d=32, scale=0.1, prefix=16, size=1 << 60):
    row = Hq * d
    cfg = skv._DECODE_CONFIG.pack(0, B, Lq, Hq, H, d, 4, 16, 4, 40, prefix, 0, scale, row * Lq, row, d, row * Lq, row, d, 4, 0, 0)
    return skv.lib().skv_attn_decode(cfg, P, P, P, P, P, None, P, None, None, P, size, None)


@pytest.mark.parametrize("B,Hq", [(8193, 8191), (2731, 3 * 8191), (62 * 601, 1801)])
def test_joins_that_no_grid_holds_are_refused(B, Hq):
    """B Lq Hq of 2^26 - 3 and more: the join's grid would have 2^32 threads."""
    assert B * Hq >= (1 << 26) - 3
    assert _size(B, 1, Hq) == skv.ERR_INVALID_ARG
    assert _decode(B, 1, Hq) == skv.ERR_INVALID_ARG


def test_the_largest_joins_are_not_refused():
    n = (1 << 26) - 4
    assert n % 1020 == 0 and _size(n // 1020, 1, 1020) == skv.OK
    assert _size(1 << 20, 1, 63) == skv.OK
    assert _size(1 << 20, 1, 64) == skv.ERR_INVALID_ARG


def _prompt(scale):
    cfg = skv._ATTN_CONFIG.pack(0, 4, 2, 64, 1, scale, 256, 64, 256, 64)
    req = skv._ATTN_REQUEST.pack(0, 0, 0, 0, 0, 0, 0, 64, 64)
    return skv.lib().skv_attn_prompt(cfg, req, 1, None, 0, None)


@pytest.mark.parametrize("scale,status", [(2.3e38, skv.OK), (2.4e38, skv.ERR_INVALID_ARG), (3.4e38, skv.ERR_INVALID_ARG)])
def test_scales_that_pass_binary32_in_base_2_are_refused(scale, status):
    """The kernels multiply by scale log2(e): an infinite one would make NaN of logits of 0."""
    assert _prompt(scale) == status
    assert _decode(0, 1, 4, scale=scale) == status
