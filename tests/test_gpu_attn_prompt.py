"""Prompt attention against its definition in float64: types, head layouts,
lengths from zero and one to several tiles, causal and not, both layouts of K
and V, strides, hidden infinities and NaN, the split form, streams and graphs."""
import numpy as np
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
