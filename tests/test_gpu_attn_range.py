"""Values of V up to the type's limit: the result is an average of them, so it is finite, however many keys
and whatever references the unnormalized sums are held against."""
import pytest
import torch

from attn_bounds import decode, prompt
from attn_reference import attention, check

pytestmark = pytest.mark.gpu
LIMIT = {torch.float16: 6.4e4, torch.bfloat16: 3.2e38}


def _inputs(nq, Hq, nk, H, d, dtype, seed, rise=5.5):
    """Logits near 0 for the first 64 keys and near `rise` (nats) for the others; V of one sign near the limit."""
    g = torch.Generator().manual_seed(seed)
    u = torch.ones(d)
    q = (u + 0.05 * torch.randn(nq, Hq, d, generator=g)).to(dtype)
    c = torch.where(torch.arange(nk) < 64, 0.0, rise / d ** 0.5)
    k = (c[:, None, None] * u + 0.02 * torch.randn(nk, H, d, generator=g)).to(dtype)
    v = (LIMIT[dtype] * (0.5 + 0.5 * torch.rand(nk, H, d, generator=g))).to(dtype)
    return q, k, v


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("nq,nk,Hq,H,split", [
    (3, 128, 4, 2, False),     # one row tile, two key streams
    (50, 700, 4, 2, False),
    (130, 1100, 2, 1, False),  # four row tiles
    (5, 4000, 2, 1, True), (130, 2100, 2, 1, True)])
def test_prompt(nq, nk, Hq, H, split, d, dtype):
    q, k, v = _inputs(nq, Hq, nk, H, d, dtype, seed=d)
    want = attention(q, k, v, torch.ones(nq, nk, dtype=torch.bool), d ** -0.5)
    assert torch.isfinite(want[0]).all()
    check(*prompt(q, k, v, [nq], [nk], is_causal=False, split=split), want, (nq, nk, d))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("count,prefix,n", [(1, 0, 200), (2, 0, 3000), (3, 640, 1400), (70, 256, 300)])
def test_decode(count, prefix, n, d, dtype):
    Hq, H = 4, 2
    g = torch.Generator().manual_seed(n)
    q, k, v = zip(*[_inputs(1, Hq, n, H, d, dtype, seed=b) for b in range(count)])
    q, k, v = torch.stack(q), torch.stack(k), torch.stack(v)
    k[:, :prefix], v[:, :prefix] = k[:1, :prefix], v[:1, :prefix]
    lens = [n - int(torch.randint(0, max(1, n - prefix), (1,), generator=g)) if b else n for b in range(count)]
    want = [attention(q[b], k[b, :m], v[b, :m], torch.ones(1, m, dtype=torch.bool), d ** -0.5) for b, m in enumerate(lens)]
    check(*decode(q, k, v, lens, prefix), tuple(torch.stack(x) for x in zip(*want)), (count, prefix, n, d))


@pytest.mark.parametrize("d", [64, 256])
def test_infinities_beside_large_values(d):
    """An infinity that a row sees reaches its channel; the other channels stay finite averages."""
    q, k, v = _inputs(130, 2, 1100, 1, d, torch.bfloat16, seed=1)
    v[1000, 0, 5], v[1099, 0, 7] = float("inf"), float("-inf")
    seen = torch.arange(1100)[None, :] <= torch.arange(130)[:, None] + 970
    check(*prompt(q, k, v, [130], [1100]), attention(q, k, v, seen, d ** -0.5), d)
