"""A row that sees keys whose logits are all -infinity is no empty row: softmax over them is NaN (exp(-inf - -inf)),
while its log-sum is -infinity; where another key's logit is finite those keys have no weight."""
import pytest
import torch

from attn_bounds import decode, prompt
from attn_reference import attention, check
from paper_2606_08635_amd import skv

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]


def _inputs(nq, Hq, nk, H, d, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(n, h, d, generator=g).to(dtype) for n, h in ((nq, Hq), (nk, H), (nk, H)))
    q[..., 0] = 1.0  # a key with -infinity there has that logit in every row
    return q, k, v


def _check(out, lse, q, k, v, seen, name):
    """seen [nq][nk]: which keys each row sees; -infinity in a key's first channel is its logit."""
    low = torch.isinf(k[:, 0, 0])
    finite = seen & ~low
    lost, none = ~finite.any(1) & seen.any(1), ~seen.any(1)
    assert torch.isnan(out[lost]).all() and (lse[lost] == -float("inf")).all(), name
    assert (out[none] == 0).all() and (lse[none] == -float("inf")).all(), name
    rows = finite.any(1)
    if rows.any():
        k = torch.where(low[:, None, None], 0.0, k.float()).to(k.dtype)
        want = attention(q, k, v, finite, q.shape[2] ** -0.5)
        check(out[rows.cuda()], lse[rows.cuda()], tuple(x[rows] for x in want), name)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("nq,nk,low,split", [
    (1, 1, 1, False), (70, 70, 40, False), (90, 70, 40, False), (130, 1100, 1050, False), (130, 1100, 1100, False),
    (5, 4000, 4000, True), (5, 4000, 3000, True), (5, 4000, 3998, True)])
def test_prompt(nq, nk, low, split, d, dtype):
    """The first `low` keys' logits are -infinity: rows that see only those, some more, none."""
    q, k, v = _inputs(nq, 2, nk, 1, d, dtype)
    k[:low, :, 0] = -float("inf")
    seen = torch.arange(nk)[None, :] <= torch.arange(nq)[:, None] + nk - nq
    _check(*prompt(q, k, v, [nq], [nk], split=split), q, k, v, seen, (nq, nk, low, d))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [32, 128, 256])
@pytest.mark.parametrize("prefix,n", [(0, 50), (0, 3000), (512, 700), (512, 3000)])
def test_decode(prefix, n, d, dtype):
    """Requests whose kept tokens have only such logits, some others, and none kept at all."""
    B, Hq, H, Lq = 4, 2, 1, 2
    q, k, v = (torch.stack(x) for x in zip(*[_inputs(Lq, Hq, n, H, d, dtype, seed=b) for b in range(B)]))
    tiers = torch.zeros(B, n, dtype=torch.uint8)
    tiers[:, 3:prefix:4] = skv.DROP
    if prefix:
        tiers[:, 0:2] = skv.DROP
    k[:, :prefix, :, 0] = -float("inf")
    k[0, :, :, 0] = -float("inf")          # all of request 0
    k[1, :n - 1, :, 0] = -float("inf")     # all but the newest of request 1
    tiers[2] = torch.where(torch.arange(n) < prefix, tiers[2], skv.DROP)  # request 2 keeps the prefix alone (or nothing)
    k[:, :prefix], v[:, :prefix] = k[:1, :prefix], v[:1, :prefix]
    lens = [n, n, n, max(prefix // 2, 1)]  # request 3 ends inside the prefix
    out, lse = decode(q, k, v, lens, prefix, tiers)
    for b, m in enumerate(lens):
        seen = torch.arange(m)[None, :] <= torch.arange(Lq)[:, None] + m - Lq
        seen = seen & (tiers[b, :m] != skv.DROP)
        _check(out[b], lse[b], q[b], k[b, :m], v[b, :m], seen, (b, prefix, n, d))
