"""Refusals and sizes of the attention and page operators that need no GPU:
every call here fails its argument check before any HIP call, or is host only."""
import ctypes
import struct

import pytest
import torch

from paper_2606_08635_amd import skv

BAD = skv.ERR_INVALID_ARG
P = 4096  # an aligned address that no refused call dereferences


@pytest.fixture(scope="module")
def lib():
    import os

    if not os.path.exists(skv.LIB_PATH):
        from paper_2606_08635_amd import build
        build.build()
    return skv.lib()


def _prompt(lib, cfg=(), req=(), count=1, ws=None, size=0):
    c = dict(dtype=0, Hq=8, H=2, d=128, causal=1, scale=0.1, qt=1024, qh=128, ot=1024, oh=128)
    c.update(cfg)
    r = dict(nq=5, nk=7, q=P, k=P, v=P, out=P, lse=0, kt=256, kh=128)
    r.update(req)
    return lib.skv_attn_prompt(skv._ATTN_CONFIG.pack(*c.values()), skv._ATTN_REQUEST.pack(*r.values()), count, ws, size, None)


@pytest.mark.parametrize("cfg", [
    dict(dtype=2), dict(dtype=-1), dict(Hq=7), dict(H=0), dict(Hq=0), dict(Hq=65540, H=65540), dict(d=96), dict(d=512),
    dict(causal=2), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(qt=1020),
    dict(qh=0), dict(ot=-8), dict(oh=4)], ids=str)
def test_prompt_configurations_refused(lib, cfg):
    assert _prompt(lib, cfg) == BAD


@pytest.mark.parametrize("req", [
    dict(nq=-1), dict(nk=-1), dict(nk=(1 << 30) + 1), dict(nq=(1 << 29)), dict(q=0), dict(q=P + 8), dict(out=0),
    dict(out=P + 2), dict(k=0), dict(v=P + 4), dict(lse=P + 2), dict(kt=0), dict(kt=1 << 25), dict(kt=12), dict(kh=-8)], ids=str)
def test_prompt_requests_refused(lib, req):
    assert _prompt(lib, req=req) == BAD


def test_prompt_other_refusals(lib):
    assert _prompt(lib, count=-1) == BAD
    assert _prompt(lib, ws=P + 8, size=1 << 20) == BAD
    cfg, req = skv._ATTN_CONFIG.pack(0, 8, 2, 128, 1, 0.1, 8, 8, 8, 8), skv._ATTN_REQUEST.pack(1, 1, P, P, P, P, 0, 8, 8)
    assert lib.skv_attn_prompt(None, req, 1, None, 0, None) == BAD
    assert lib.skv_attn_prompt(cfg, None, 1, None, 0, None) == BAD
    assert lib.skv_attn_prompt(cfg, None, 0, None, 0, None) == skv.OK  # nothing to do
    assert lib.skv_attn_prompt_workspace_size(cfg, req, 1, None) == BAD


def test_prompt_workspace_size(lib):
    size = skv.attn_prompt_workspace_size
    assert size([8000], [8000], 32, 8, 128) == 0  # enough workgroups as it is
    assert size([100], [1000], 32, 8, 128) == 0  # too short to cut
    parts = size([100], [30000], 32, 8, 128) / (100 * 32 * (128 + 2) * 4)
    assert parts == int(parts) and 2 <= parts <= 64
    assert size([], [], 32, 8, 128) == 0
    with pytest.raises(skv.SkvError):
        size([1], [1], 32, 7, 128)
    with pytest.raises(ValueError):
        size([1, 2], [1], 32, 8, 128)


def _decode(lib, ptrs=(), ws=P, size=1 << 30, **cfg):
    c = dict(dtype=0, B=3, Lq=1, Hq=8, H=2, d=128, nb=100, bs=16, width=10, max_len=100, prefix=0, tier_len=0, scale=0.1,
             qr=1024, qt=1024, qh=128, orr=1024, ot=1024, oh=128, ts=10, tr=0, th=0)
    c.update(cfg)
    p = dict(q=P, k=P, v=P, tables=P, lens=P, tiers=None, out=P, lse=None, status=None)
    p.update(ptrs)
    return lib.skv_attn_decode(skv._DECODE_CONFIG.pack(*c.values()), *p.values(), ws, size, None)


@pytest.mark.parametrize("cfg", [
    dict(dtype=2), dict(B=-1), dict(Lq=-1), dict(Hq=9), dict(d=48), dict(nb=0), dict(bs=0), dict(nb=1 << 20, bs=1 << 12),
    dict(width=-1), dict(ts=9), dict(max_len=-1), dict(prefix=8), dict(prefix=176), dict(prefix=-16), dict(scale=0.0),
    dict(scale=float("nan")), dict(qr=4), dict(oh=0), dict(B=1 << 20, Lq=2), dict(width=1 << 27, ts=1 << 27)], ids=str)
def test_decode_configurations_refused(lib, cfg):
    assert _decode(lib, **cfg) == BAD


@pytest.mark.parametrize("ptrs", [dict(q=0), dict(k=P + 8), dict(v=0), dict(tables=P + 2), dict(lens=0), dict(out=P + 4),
                                  dict(lse=P + 1), dict(status=P + 3)], ids=str)
def test_decode_pointers_refused(lib, ptrs):
    assert _decode(lib, ptrs) == BAD


def test_decode_other_refusals(lib):
    assert _decode(lib, max_len=1000, size=0) == skv.ERR_CAPACITY
    assert _decode(lib, max_len=1000, ws=None) == BAD
    assert _decode(lib, dict(tiers=P), tier_len=-1) == BAD
    assert _decode(lib, dict(tiers=P), tier_len=5, th=-1) == BAD
    assert _decode(lib, B=0) == skv.OK
    assert _decode(lib, Lq=0) == skv.OK
    with pytest.raises(skv.SkvError):
        skv.attn_decode_workspace_size(1, 1, 8, 3, 128, 100)


def test_decode_workspace_size(lib):
    size = skv.attn_decode_workspace_size
    assert size(3, 1, 8, 2, 128, 200) == 0  # short requests are written at once
    assert size(2, 1, 8, 2, 128, 5000) > 0
    # a part holds every row's sums, reference and sum
    one = size(1, 1, 8, 2, 128, 5000) - 8
    assert one % (8 * (128 + 2) * 4) == 0


POOL = dict(L=2, nb=10, bs=4, row=512, k=P, v=P, refs=P)


def _pool(**kw):
    return skv._PAGE_POOL.pack(*dict(POOL, **kw).values())


@pytest.mark.parametrize("pool", [dict(L=0), dict(nb=0), dict(bs=0), dict(nb=1 << 20, bs=1 << 12), dict(row=8), dict(row=24),
                                  dict(k=0), dict(v=P + 8), dict(refs=0), dict(refs=P + 4)], ids=str)
def test_page_pools_refused(lib, pool):
    p, ws = _pool(**pool), 1 << 20
    assert lib.skv_pages_fork(p, P, 3, P, 2, P, 2, P, 3, P, P, P, ws, None) == BAD
    assert lib.skv_pages_compact(p, P, 3, P, 2, P, 12, 12, P, 3, P, P, P, ws, None) == BAD
    if not {"k", "v"} & set(pool):
        assert lib.skv_pages_reserve(p, P, 3, P, P, 2, P, P, ws, None) == BAD
        assert lib.skv_pages_free(p, P, 3, P, 2, P, None) == BAD
    if "refs" not in pool:
        assert lib.skv_pages_copy(p, _pool(), P, P, 1, P, None) == BAD
        assert lib.skv_pages_copy(_pool(), p, P, P, 1, P, None) == BAD


def test_page_arguments_refused(lib):
    p, ws = _pool(), 1 << 20
    fork = lib.skv_pages_fork
    assert fork(None, P, 3, P, 2, P, 2, P, 3, P, P, P, ws, None) == BAD
    assert fork(p, P, 3, P, -1, P, 2, P, 3, P, P, P, ws, None) == BAD
    assert fork(p, P, -1, P, 2, P, 2, P, 3, P, P, P, ws, None) == BAD
    assert fork(p, 0, 3, P, 2, P, 2, P, 3, P, P, P, ws, None) == BAD
    assert fork(p, P, 3, P, 2, 0, 2, P, 3, P, P, P, ws, None) == BAD
    assert fork(p, P, 3, P, 2, P, 2, P, 3, P, 0, P, ws, None) == BAD
    assert fork(p, P, 3, P, 2, P, 2, P, 3, P, P, 0, ws, None) == BAD
    assert fork(p, P, 3, P, 2, P, 2, P, 3, P, P, P, 16, None) == skv.ERR_CAPACITY
    compact = lib.skv_pages_compact
    assert compact(p, P, 3, P, 2, 0, 12, 12, P, 3, P, P, P, ws, None) == BAD
    assert compact(p, P, 3, P, 2, P, -1, 12, P, 3, P, P, P, ws, None) == BAD
    assert compact(p, P, 3, P, 2, P, 12, -1, P, 3, P, P, P, ws, None) == BAD
    assert lib.skv_pages_reserve(p, P, 3, P, 0, 2, P, P, ws, None) == BAD
    assert lib.skv_pages_free(p, P, 3, P, 2, 0, None) == BAD
    copy = lib.skv_pages_copy
    assert copy(p, _pool(L=3), P, P, 1, P, None) == BAD
    assert copy(p, _pool(bs=8), P, P, 1, P, None) == BAD
    assert copy(p, _pool(row=528), P, P, 1, P, None) == BAD
    assert copy(p, p, P, P, -1, P, None) == BAD
    assert copy(p, p, 0, P, 1, P, None) == BAD
    out = ctypes.c_uint64()
    for args in ((-1, 10, 5), (1, 0, 5), (1, 10, -1)):
        assert lib.skv_pages_workspace_size(*args, ctypes.byref(out)) == BAD
    # tables of up to 1024 tokens a page fit what their requests' lengths ask for
    a, b = skv.pages_workspace_size(4, 100, 1000), skv.pages_workspace_size(4, 100, 2000)
    assert 0 < a <= b


def test_structures_are_the_headers(tmp_path):
    """The binding's packed structures have the header's sizes."""
    import os
    import subprocess

    from paper_2606_08635_amd import build as B

    if not os.path.exists(B.HIPCC):
        pytest.skip("hipcc not found")
    src, exe = tmp_path / "sizes.cpp", str(tmp_path / "sizes")
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "skv.h"\nint main() { printf("%zu %zu %zu %zu %zu %zu",'
                   "sizeof(skv_attn_config), sizeof(skv_attn_request), sizeof(skv_decode_config), sizeof(skv_page_pool),"
                   "offsetof(skv_decode_config, q_request_stride), offsetof(skv_attn_request, kv_token_stride)); }")
    subprocess.run([B.HIPCC, "-I", B.INCLUDE, str(src), "-o", exe], check=True, capture_output=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == [skv._ATTN_CONFIG.size, skv._ATTN_REQUEST.size, skv._DECODE_CONFIG.size, skv._PAGE_POOL.size,
                   struct.calcsize("@12if0q"), struct.calcsize("@2i5P")]


def test_host_tensors_refused():
    x = torch.zeros(4, 2, 64, dtype=torch.float16)
    with pytest.raises(ValueError):
        skv.attn_prompt(x, x, x, x)
    with pytest.raises(TypeError):
        skv.attn_prompt(x.float(), x, x, x)
    c, t = torch.zeros(3, 16, 2, 64, dtype=torch.float16), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(ValueError):
        skv.attn_decode(x[None], c, c, t, t[0], x[None], None, 4)
    with pytest.raises(ValueError):
        skv.pages_free(t[0], t, t[0], 16, t[0])


def test_sizes_past_the_limits_refused(lib):
    """Just past what a launch and the kernels' indexes hold: refused by the host."""
    assert _decode(lib, B=1 << 10, Lq=1 << 10, Hq=64, H=64) == BAD
    assert _decode(lib, width=(1 << 26) + 1, ts=(1 << 26) + 1) == BAD
    assert _decode(lib, B=1 << 19, Hq=8, H=8, max_len=10) == skv.ERR_CAPACITY
    # 48 small requests and one that no grid holds: nothing of it is launched
    cfg = skv._ATTN_CONFIG.pack(0, 4096, 4096, 32, 1, 0.1, 1 << 17, 32, 1 << 17, 32)
    small, huge = (skv._ATTN_REQUEST.pack(n, n, P, P, P, P, 0, 1 << 17, 32) for n in (1, 1 << 20))
    assert lib.skv_attn_prompt(cfg, small * 48 + huge, 49, None, 0, None) == skv.ERR_CAPACITY
    p, ws = _pool(), 1 << 40
    assert lib.skv_pages_free(p, P, 0, P, (1 << 24) + 1, P, None) == BAD
    assert lib.skv_pages_reserve(p, P, 0, P, P, (1 << 24) + 1, P, P, ws, None) == BAD


@pytest.mark.parametrize("out,out_lens,fork_only", [
    (0x10000, 0x90000, False),         # the tables themselves
    (0x10000 + 20, 0x90000, False),    # their last entry
    (0x80000, 0x20000, False),         # the lengths themselves
    (0x20000 - 8, 0x90000, False), (0x80000, 0x10008, False), (0x80000, 0x80000 + 8, False),
    (0x30000, 0x90000, True), (0x80000, 0x30000, True)])  # the parents
def test_outputs_on_inputs_refused(lib, out, out_lens, fork_only):
    """Fork and compact read their inputs until their last launch."""
    p, ws = _pool(), 1 << 20
    tables, lens, parents = 0x10000, 0x20000, 0x30000
    assert lib.skv_pages_fork(p, tables, 3, lens, 2, parents, 2, out, 3, out_lens, P, P, ws, None) == BAD
    if not fork_only:
        assert lib.skv_pages_compact(p, tables, 3, lens, 2, P, 12, 12, out, 3, out_lens, P, P, ws, None) == BAD
