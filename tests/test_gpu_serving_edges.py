"""Calls that the documentation allows beside the usual ones: padded batches, a first request that is empty or ends
inside the shared prefix, compaction of forks that share their pages, one request released from several tables."""
import pytest
import torch

from attn_reference import attention, causal, check
from paper_2606_08635_amd import skv

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("first", [0, 3, 200])
@pytest.mark.parametrize("d", [64, 256])
def test_first_request_short_and_padded_batch(d, first):
    """The prefix is read through request 0's table whatever its length; empty requests' tables behind it are not read."""
    B, Hq, H, block, prefix, n, Lq = 5, 4, 2, 16, 512, 700, 2
    g = torch.Generator().manual_seed(d + first)
    width, shared = -(-n // block), prefix // block
    blocks = shared + B * (width - shared)
    tables = torch.cat([torch.arange(shared).expand(B, shared),
                        shared + torch.arange(B * (width - shared)).view(B, -1)], 1).int().contiguous()
    k, v = (torch.randn(blocks * block, H, d, generator=g).half() for _ in range(2))
    q = torch.randn(B, Lq, Hq, d, generator=g).half()
    lens = [first, n, 0, 650, 0]
    tables[2], tables[4] = -1, 1 << 30  # slots without a request
    tables[0, shared:] = -7             # nothing of it is in use past the prefix
    want = []
    for b, m in enumerate(lens):
        t = torch.arange(m)
        rows = tables[b, t // block].long() * block + t % block
        want.append(attention(q[b], k[rows], v[rows], causal(Lq, m), d ** -0.5))
    want = tuple(torch.stack(x) for x in zip(*want))
    ws = torch.empty(skv.attn_decode_workspace_size(B, Lq, Hq, H, d, n, prefix), dtype=torch.uint8, device=DEV)
    out, lse = torch.full((B, Lq, Hq, d), 7.0, dtype=torch.float16, device=DEV), torch.full((B, Lq, Hq), 7.0, device=DEV)
    bad = torch.zeros(1, dtype=torch.int32, device=DEV)
    cache = [x.view(blocks, block, H, d).to(DEV) for x in (k, v)]
    skv.attn_decode(q.to(DEV), *cache, tables.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), out, ws, n,
                    prefix_len=prefix, lse=lse, dev_status=bad)
    check(out, lse, want, (d, first))
    assert bad.item() == 0


def test_compaction_of_forks_and_their_release():
    """Three forks of a request compacted at once by maps of their own, then everything released."""
    L, H, d, block, n, nb, B = 2, 2, 64, 16, 200, 120, 3
    g = torch.Generator(device=DEV).manual_seed(4)
    k, v = (torch.randn(L, nb, block, H, d, generator=g, device=DEV).half() for _ in range(2))
    width = -(-n // block)
    refs = torch.zeros(nb, dtype=torch.int32, device=DEV)
    ws = torch.empty(skv.pages_workspace_size(B, nb, width * block), dtype=torch.uint8, device=DEV)
    st = torch.full((1,), -1, dtype=torch.int32, device=DEV)
    table, lens = torch.full((1, width), -1, dtype=torch.int32, device=DEV), torch.tensor([n], dtype=torch.int32, device=DEV)
    skv.pages_reserve(refs, table, torch.zeros_like(lens), lens, block, ws, st)
    kids, kid_lens = torch.full((B, width), -1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    skv.pages_fork(k, v, refs, table, lens, torch.zeros(B, dtype=torch.int32, device=DEV), kids, kid_lens, ws, st)
    assert st.item() == 0 and refs.max().item() == B + 1
    tiers = torch.zeros(B, n, dtype=torch.uint8, device=DEV)
    tiers[0, 100::3], tiers[1, 5:9], tiers[2] = skv.DROP, skv.DROP, skv.DROP
    small, small_lens = torch.full_like(kids, -1), torch.zeros_like(kid_lens)
    skv.pages_compact(k, v, refs, kids, kid_lens, tiers, small, small_lens, ws, st)
    assert st.item() == 0
    at = torch.arange(n, device=DEV)
    for b in range(B):
        keep = at[tiers[b] != skv.DROP]
        to = torch.arange(len(keep), device=DEV)
        assert small_lens[b].item() == len(keep)
        for x in (k, v):
            assert torch.equal(x[:, small[b].long()[to // block], to % block], x[:, kids[b].long()[keep // block], keep % block])
    assert torch.equal(small[0, :100 // block], kids[0, :100 // block])
    # the children twice in one call: once more than they are held
    twice, twice_lens = torch.cat([kids, kids]), torch.cat([kid_lens, kid_lens])
    skv.pages_free(refs, small, small_lens, block, st)
    assert st.item() == 0
    skv.pages_free(refs, table, lens, block, st)
    assert st.item() == 0
    skv.pages_free(refs, twice, twice_lens, block, st)
    assert st.item() == skv.ERR_FORMAT  # more entries than counts: the rest is released all the same
    assert (refs == 0).all()
