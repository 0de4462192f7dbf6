"""Many keys of small probability behind one large one whose V is zero: together they are the whole result, so none of
them may be lost.  In binary16 a probability is held to 2^-33 of the row's largest, in bfloat16 to far less."""
import pytest
import torch

from attn_bounds import bound, decode, prompt, within
from attn_reference import HALF_STEP

pytestmark = pytest.mark.gpu
TINY = {torch.float16: 2.0 ** -33, torch.bfloat16: 0.0}


def _inputs(nq, Hq, nk, H, d, dtype, below, seed=0):
    """Logits: `below` (in powers of two) less than the first key's, within about 0.05; the first key's V is 0."""
    g = torch.Generator().manual_seed(seed)
    scale = d ** -0.5
    q = torch.ones(nq, Hq, d).to(dtype)
    k = 0.02 * torch.randn(nk, H, d, generator=g)
    k[0] += below * 0.6931471805599453 / (d * scale)
    v = 0.5 + torch.rand(nk, H, d, generator=g)
    v[0] = 0
    return q, k.to(dtype), v.to(dtype)


def _want(q, k, v, scale):
    G = q.shape[1] // k.shape[1]
    kh, vh = (x.double().repeat_interleave(G, 1).transpose(0, 1) for x in (k, v))
    z = q.double().transpose(0, 1) @ kh.transpose(1, 2).contiguous() * scale
    return (torch.softmax(z, 2) @ vh).transpose(0, 1)


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("nq,Hq,H,nk,split", [(2, 2, 1, 1000, False), (130, 1, 1, 32768, False), (4, 2, 2, 32768, True)])
def test_prompt(nq, Hq, H, nk, split, d, dtype):
    for below in (12.5, 25.5, 28.5):
        q, k, v = _inputs(nq, Hq, nk, H, d, dtype, below)
        want = _want(q, k, v, d ** -0.5)
        tol = bound(q, k, v, torch.ones(nq, nk, dtype=torch.bool), d ** -0.5, want, HALF_STEP[dtype], TINY[dtype])
        assert (tol < want / 2).all()  # a result that lost them is seen
        out, _ = prompt(q, k, v, [nq], [nk], is_causal=False, split=split)
        within(out, want, tol, (nq, nk, d, below))


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
@pytest.mark.parametrize("prefix,n", [(0, 200), (0, 32768), (16384, 16500)])
def test_decode(prefix, n, d, dtype):
    for below in (12.5, 25.5, 28.5):
        q, k, v = _inputs(1, 2, n, 1, d, dtype, below, seed=1)
        want = _want(q, k, v, d ** -0.5)
        tol = bound(q, k, v, torch.ones(1, n, dtype=torch.bool), d ** -0.5, want, HALF_STEP[dtype], TINY[dtype])
        assert (tol < want / 2).all()
        out, _ = decode(q[None].expand(2, -1, -1, -1).contiguous(), torch.stack([k, k]), torch.stack([v, v]), [n, n], prefix)
        for b in range(2):
            within(out[b], want, tol, (prefix, n, d, below))
