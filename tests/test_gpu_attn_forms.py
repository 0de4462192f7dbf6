"""Forms of the attention kernels that sizes select and that the other tests do not reach together with values that are
not finite, rows without keys, shared and unshared prefixes, and the second term of the probabilities."""
import pytest
import torch

from attn_bounds import bound, decode, prompt, within
from attn_reference import HALF_STEP, attention, causal, check
from paper_2606_08635_amd import skv

pytestmark = pytest.mark.gpu
TYPES = [torch.float16, torch.bfloat16]


def _random(nq, Hq, nk, H, d, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    return tuple(torch.randn(n, h, d, generator=g).to(dtype) for n, h in ((nq, Hq), (nk, H), (nk, H)))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_hidden_values_with_four_row_tiles(d, dtype):
    """More than 1024 keys and 128 rows: workgroups of 128 rows.  Infinities and NaN in V and K reach the rows that see
    their keys and no other, in the last tiles and in ones that every row sees."""
    nq, nk = 150, 1100
    q, k, v = _random(nq, 2, nk, 1, d, dtype, d)
    # seen by the last 20, 60 and 100 queries, and by every query
    v[nk - 20, 0, 1], v[nk - 20, 0, 2], v[nk - 60, 0, d - 1] = float("inf"), float("nan"), float("-inf")
    v[nk - 100, 0, 3], v[400, 0, 4], v[401, 0, 4], v[402, 0, 5] = float("inf"), float("inf"), float("-inf"), float("nan")
    k[nk - 10, 0, :] = float("nan")
    want = attention(q, k, v, causal(nq, nk), d ** -0.5)
    check(*prompt(q, k, v, [nq], [nk]), want, d)


@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_rows_without_keys_with_four_row_tiles(d):
    nq, nk = 1500, 1100
    q, k, v = _random(nq, 1, nk, 1, d, torch.float16, d)
    v[0, 0, 0] = float("nan")
    out, lse = prompt(q, k, v, [nq], [nk])
    assert (out[:400] == 0).all() and (lse[:400] == -float("inf")).all()
    check(out, lse, attention(q, k, v, causal(nq, nk), d ** -0.5), d)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [64, 256])
def test_hidden_values_in_a_prefix_of_many_rows(d, dtype):
    """40 requests of two rows behind a prefix: its workgroups have three and four row tiles' places."""
    B, n, prefix = 40, 330, 320
    g = torch.Generator().manual_seed(d)
    q, k, v = (torch.randn(B, m, h, d, generator=g).to(dtype) for m, h in ((1, 4), (n, 2), (n, 2)))
    k[:, :prefix], v[:, :prefix] = k[:1, :prefix], v[:1, :prefix]
    tiers = torch.zeros(B, n, dtype=torch.uint8)
    tiers[:, 5:prefix:3] = skv.DROP
    v[:, 5:prefix:3], k[:, 8:prefix:3] = float("nan"), float("inf")
    lens = [n - b % 7 for b in range(B)]
    lens[3], lens[11] = 200, 1          # inside the prefix
    v[:, 300, 1, 2] = float("-inf")     # in the prefix, seen by all but those
    v[5, n - 6, 0, 1] = float("inf")    # in one request's own
    tiers[:, 300] = 0
    out, lse = decode(q, k, v, lens, prefix, tiers)
    for b, m in enumerate(lens):
        seen = (tiers[b, :m] != skv.DROP)[None]
        check(out[b], lse[b], attention(q[b], k[b, :m], v[b, :m], seen, d ** -0.5), (b, d))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("count,Lq", [(3, 1), (9, 2), (40, 4)])
def test_prefix_shared_and_not(count, Lq, d):
    """One batch with its prefix read once and read by every request; one request ends inside it."""
    g = torch.Generator().manual_seed(count)
    n = 448 + 7 * count
    q, k, v = (torch.randn(count, m, h, d, generator=g).half() for m, h in ((Lq, 4), (n, 2), (n, 2)))
    k[:, :448], v[:, :448] = k[:1, :448], v[:1, :448]
    lens = [448 + 7 * i for i in range(count)]
    lens[1], lens[-1] = 100, 448
    want = [attention(q[b], k[b, :m], v[b, :m], causal(Lq, m), d ** -0.5) for b, m in enumerate(lens)]
    want = tuple(torch.stack(x) for x in zip(*want))
    check(*decode(q, k, v, lens, 448), want, "shared")
    check(*decode(q, k, v, lens, 0), want, "unshared")


def _cancelling(nq, Hq, nk, H, d, dtype, seed):
    """Logits that binary32 holds exactly (queries of one channel), a few keys of weight, and in each KV head a last key
    that takes back what the others add up to, so that the results are small and their rounding hides no error of the
    probabilities."""
    q, k, v = _random(nq, Hq, nk, H, d, dtype, seed)
    g = torch.Generator().manual_seed(seed + 1)
    q[:] = 0
    q[..., 3] = 1
    k[..., 3] = (-min(nk / 4, 60.0) * torch.rand(nk, H, generator=g) * d ** 0.5).to(dtype)
    k[0, :, 3] = k[-1, :, 3] = -0.4 * d ** 0.5
    for h in range(H):
        p = torch.softmax(k[:, h, 3].double() * d ** -0.5, 0)
        v[-1, h] = (-(p[:-1] @ v[:-1, h].double()) / p[-1]).to(dtype)
    return q, k, v


def _two_terms(out, q, k, v, name):
    """Within a bound that two-term probabilities keep and one-term ones would not (shown by rounding them here)."""
    nq, Hq, d = q.shape
    nk, H, _ = k.shape
    t = q.dtype
    scale = d ** -0.5
    want, one = (torch.zeros(nq, Hq, d, dtype=torch.float64) for _ in range(2))
    for h in range(Hq):
        kh, vh = k[:, h // (Hq // H)].double(), v[:, h // (Hq // H)].double()
        z = q[:, h].double() @ kh.t() * scale
        e = torch.exp(z - z.amax(1, keepdim=True))
        want[:, h] = e @ vh / e.sum(1, keepdim=True)
        one[:, h] = e.to(t).double() @ vh / e.sum(1, keepdim=True)
    # what a rounding leaves over is itself rounded: half a step of half a step; below binary16's range by 2^-25
    tol = bound(q, k, v, torch.ones(nq, nk, dtype=torch.bool), scale, want, HALF_STEP[t] ** 2,
                2.0 ** -25 if t == torch.float16 else 0.0, dots=8)
    lost = ((one - want).abs() > tol).double().mean()
    assert lost > 0.25, (name, lost)
    within(out, want, tol, name)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [64, 128, 256])
def test_second_term_in_cut_tiles(d, dtype):
    """Prompts whose only tile the end of the keys cuts."""
    for nq, nk in ((1, 20), (40, 30)):
        q, k, v = _cancelling(nq, 4, nk, 4, d, dtype, seed=nk)
        out, _ = prompt(q, k, v, [nq], [nk], is_causal=False)
        _two_terms(out, q, k, v, (nq, nk, d))


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("n", [64, 256, 512])
def test_second_term_in_decode(n, d, dtype):
    """Whole tiles of a request's own tokens, with one row tile and with two."""
    for Hq, H in ((4, 4), (40, 1)):
        q, k, v = _cancelling(1, Hq, n, H, d, dtype, seed=n)
        out, _ = decode(q[None], k[None], v[None], [n])
        _two_terms(out[0], q, k, v, (n, d, Hq))
