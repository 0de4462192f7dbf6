"""Prompt attention against its definition in float64: types, head layouts,
lengths from zero and one to several tiles, causal and not, both layouts of K
and V, strides, hidden infinities and NaN, the split form, streams and graphs."""
import pytest
import torch

from attn_reference import attention, causal, check
from paper_2606_08635_amd import skv

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float16, torch.bfloat16]


def _inputs(ql, kl, Hq, H, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(sum(ql), Hq, d, generator=g).to(dtype)
    k = torch.randn(sum(kl), H, d, generator=g).to(dtype)
    v = torch.randn(sum(kl), H, d, generator=g).to(dtype)
    return q, k, v


def _reference(q, k, v, ql, kl, is_causal, scale):
    parts, qo, ko = [], 0, 0
    for nq, nk in zip(ql, kl):
        seen = causal(nq, nk) if is_causal else torch.ones(nq, nk, dtype=torch.bool)
        parts.append(attention(q[qo:qo + nq], k[ko:ko + nk], v[ko:ko + nk], seen, scale))
        qo, ko = qo + nq, ko + nk
    return tuple(torch.cat(x) for x in zip(*parts))


def _run(q, k, v, ql, kl, is_causal=True, ws=None, **kw):
    qd, kd, vd = q.to(DEV), k.to(DEV), v.to(DEV)
    out = torch.full_like(qd, 7.0)
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device=DEV)
    skv.attn_prompt(qd, kd, vd, out, ql, kl, causal=is_causal, lse=lse, ws=ws, **kw)
    torch.cuda.synchronize()
    return out, lse


HEADS = [(4, 2), (7, 1), (2, 2), (32, 8)]


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("is_causal", [True, False])
def test_ragged_sequences(d, dtype, is_causal):
    for Hq, H in HEADS[:3]:
        ql, kl = [1, 65, 0, 200, 33], [1, 65, 5, 200, 161]
        q, k, v = _inputs(ql, kl, Hq, H, d, dtype, seed=d)
        got = _run(q, k, v, ql, kl, is_causal)
        check(*got, _reference(q, k, v, ql, kl, is_causal, d ** -0.5), (Hq, H, d))


@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 64), (1, 65), (2, 1), (5, 3), (64, 64), (63, 129), (300, 100), (3, 0), (128, 1000)])
@pytest.mark.parametrize("is_causal", [True, False])
def test_lengths(nq, nk, is_causal):
    """Queries past the keys included: the first ones see nothing."""
    for d, (Hq, H) in ((128, (4, 2)), (64, (3, 1))):
        q, k, v = _inputs([nq], [nk], Hq, H, d, torch.float16, seed=nq + nk)
        check(*_run(q, k, v, [nq], [nk], is_causal), _reference(q, k, v, [nq], [nk], is_causal, d ** -0.5), (d, nq, nk))


@pytest.mark.parametrize("d", [64, 128, 256])
def test_long_rows(d):
    """Enough rows and keys that workgroups of four row tiles run, with references raised many times."""
    ql, kl = [1100], [1500]
    q, k, v = _inputs(ql, kl, 16, 8, d, torch.float16, seed=d)
    k *= torch.linspace(0.2, 4.0, 1500)[:, None, None].to(k.dtype)
    check(*_run(q, k, v, ql, kl), _reference(q, k, v, ql, kl, True, d ** -0.5), d)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_hidden_values_have_no_effect(d, dtype):
    """Infinities and NaN in V and K reach the rows that see their keys and no other."""
    for ql, kl, Hq, H in (([70, 3, 130], [70, 90, 130], 4, 2), ([600], [700], 16, 8)):
        q, k, v = _inputs(ql, kl, Hq, H, d, dtype, seed=d)
        n = sum(kl)
        v[30, 0, 1], v[31, 0, 1], v[40, :, 3] = float("inf"), float("-inf"), float("-inf")
        v[n - 1, 0, 0], v[n - 2, H - 1, d - 1] = float("nan"), float("inf")
        v[n - 20, 0, :] = float("nan")
        k[n - 10, H - 1, :] = float("nan")
        check(*_run(q, k, v, ql, kl), _reference(q, k, v, ql, kl, True, d ** -0.5), (d, ql))


def test_no_visible_keys_and_masks():
    """Every key hidden, whatever it holds: zeros and -infinity."""
    q, k, v = _inputs([9], [4], 4, 2, 64, torch.float16)
    v[:], k[:] = float("nan"), float("nan")
    out, lse = _run(q, k, v, [9], [4])
    assert (out[:5] == 0).all() and (lse[:5] == -float("inf")).all()
    assert torch.isnan(out[5:]).all() and torch.isnan(lse[5:]).all()


@pytest.mark.parametrize("scale", [1e-3, 1.0, 30.0])
def test_logits_of_any_size(scale):
    """References that are raised often, and logits far below the maximum."""
    q, k, v = _inputs([200], [333], 4, 2, 128, torch.float16, seed=2)
    k *= torch.linspace(0.01, 3.0, 333)[:, None, None].half()
    check(*_run(q, k, v, [200], [333], scale=scale), _reference(q, k, v, [200], [333], True, scale), scale)


@pytest.mark.parametrize("d", [64, 128, 256])
def test_codec_layout_and_strides(d):
    """K and V as [H][n][d] buffers; q and out as slices of wider tensors; packed K and V inside a fused tensor."""
    Hq, H, ql, kl = 8, 2, [33, 130], [64, 130]
    q, k, v = _inputs(ql, kl, Hq, H, d, torch.float16, seed=d)
    want = _reference(q, k, v, ql, kl, True, d ** -0.5)
    lists = [[x.transpose(0, 1).contiguous().to(DEV) for x in t.split(kl)] for t in (k, v)]
    out = torch.full((sum(ql), Hq, d), 7.0, dtype=torch.float16, device=DEV)
    lse = torch.empty(sum(ql), Hq, device=DEV)
    skv.attn_prompt(q.to(DEV), *lists, out, ql, lse=lse)
    check(out, lse, want, "lists")
    fused = torch.full((sum(kl), Hq + 2 * H, d), 7.0, dtype=torch.float16, device=DEV)
    fused[:, Hq:Hq + H], fused[:, Hq + H:] = k.to(DEV), v.to(DEV)
    fused[:sum(ql), :Hq] = q.to(DEV)
    wide = torch.full((sum(ql), Hq + 3, d + 8), 7.0, dtype=torch.float16, device=DEV)
    skv.attn_prompt(fused[:sum(ql), :Hq], fused[:, Hq:Hq + H], fused[:, Hq + H:], wide[:, 1:Hq + 1, :d], ql, kl, lse=lse)
    torch.cuda.synchronize()
    check(wide[:, 1:Hq + 1, :d], lse, want, "strided")
    wide[:, 1:Hq + 1, :d] = 7.0
    assert (wide == 7.0).all()  # nothing outside was written


@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_split_keys(d):
    """Few queries over many keys, with a workspace and without; the workspace's contents do not matter."""
    ql, kl, Hq, H = [5, 0, 40], [4000, 700, 2500], 8, 2
    q, k, v = _inputs(ql, kl, Hq, H, d, torch.bfloat16, seed=d)
    need = skv.attn_prompt_workspace_size(ql, kl, Hq, H, d)
    assert need > 0
    want = _reference(q, k, v, ql, kl, True, d ** -0.5)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)
    check(*_run(q, k, v, ql, kl, ws=ws), want, "split")
    check(*_run(q, k, v, ql, kl, ws=ws[:need - 16].clone()), want, "too small: unsplit")
    check(*_run(q, k, v, ql, kl), want, "none")


def test_more_requests_than_a_launch_takes():
    ql = [1 + 7 * i % 40 for i in range(110)]
    q, k, v = _inputs(ql, ql, 4, 2, 64, torch.float16, seed=9)
    check(*_run(q, k, v, ql, ql), _reference(q, k, v, ql, ql, True, 0.125))


def test_stream_and_graph():
    """On a stream of its own; captured and replayed with new inputs and other work between."""
    ql, kl = [300, 20], [300, 2000]
    q, k, v = (x.to(DEV) for x in _inputs(ql, kl, 8, 2, 128, torch.float16))
    ws = torch.empty(skv.attn_prompt_workspace_size(ql, kl, 8, 2, 128), dtype=torch.uint8, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        skv.attn_prompt(q, k, v, out, ql, kl, lse=lse, ws=ws)
    s.synchronize()
    first = out.clone()
    skv.attn_prompt(q, k, v, out, ql, kl, lse=lse, ws=ws, stream=s)
    s.synchronize()
    assert torch.equal(out, first)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        skv.attn_prompt(q, k, v, out, ql, kl, lse=lse, ws=ws)
    for seed in range(3):
        for x, y in zip((q, k, v), _inputs(ql, kl, 8, 2, 128, torch.float16, seed=10 + seed)):
            x.copy_(y)
        want, want_lse = torch.empty_like(out), torch.empty_like(lse)
        skv.attn_prompt(q, k, v, want, ql, kl, lse=want_lse, ws=torch.empty_like(ws))
        torch.cuda.synchronize()
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
