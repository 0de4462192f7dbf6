"""Strides at the ends of what prompt attention takes: offsets of K, V, queries and results past 32 bits."""
import pytest
import torch

from attn_reference import attention, causal, check
from paper_2606_08635_amd import skv

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _values(nq, Hq, nk, H, d):
    g = torch.Generator().manual_seed(nk)
    return tuple(torch.randn(n, h, d, generator=g).half() for n, h in ((nq, Hq), (nk, H), (nk, H)))


@pytest.mark.parametrize("d", [64, 256])
def test_largest_token_stride(d):
    """64 tokens of a tile span nearly 4 GiB; the second tile begins past it."""
    nq, nk, Hq, H, step = 5, 70, 4, 2, (1 << 25) - 8
    q, k, v = _values(nq, Hq, nk, H, d)
    pool = torch.empty(nk * step, dtype=torch.float16, device=DEV)
    kd, vd = (pool[at:].as_strided((nk, H, d), (step, d, 1)) for at in (0, 4096))
    kd.copy_(k), vd.copy_(v)
    out, lse = torch.full((nq, Hq, d), 7.0, dtype=torch.float16, device=DEV), torch.full((nq, Hq), 7.0, device=DEV)
    skv.attn_prompt(q.to(DEV), kd, vd, out, [nq], [nk], lse=lse)
    check(out, lse, attention(q, k, v, causal(nq, nk), d ** -0.5), d)
    with pytest.raises(skv.SkvError):
        far = pool.as_strided((2, H, d), (1 << 25, d, 1))
        skv.attn_prompt(q.to(DEV), far, far, out, [nq], [2])


def test_heads_queries_and_results_far_apart():
    nq, nk, Hq, H, d, step = 3, 130, 4, 2, 128, (1 << 31) + 8
    q, k, v = _values(nq, Hq, nk, H, d)
    pool = torch.empty(step + (1 << 20), dtype=torch.float16, device=DEV)
    kd, vd = (pool[at:].as_strided((H, nk, d), (step, d, 1)) for at in (0, 1 << 18))
    kd.copy_(k.transpose(0, 1)), vd.copy_(v.transpose(0, 1))
    qd, out = (pool[at:].as_strided((nq, Hq, d), ((1 << 30) + 8, d, 1)) for at in (1 << 19, (1 << 19) + 4096))
    qd.copy_(q)
    lse = torch.full((nq, Hq), 7.0, device=DEV)
    skv.attn_prompt(qd, [kd], [vd], out, [nq], lse=lse)
    check(out, lse, attention(q, k, v, causal(nq, nk), d ** -0.5))
