"""Decode attention over a paged cache against its definition in float64:
types, head layouts, drafted tokens, block sizes, shared prefixes, dropped
tokens, empty and short requests, bad tables, streams and graphs."""
import pytest
import torch

from attn_reference import attention, check
from paper_2606_08635_amd import skv

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Batch:
    """Requests in a paged cache: the rows outside their tokens hold NaN."""

    def __init__(self, lens, Hq, H, d, Lq=1, block=16, prefix=0, dtype=torch.float16, seed=0, tier_len=0, drop=0.0,
                 head_maps=False, spare=3):
        g = torch.Generator().manual_seed(seed)
        self.lens, self.Lq, self.prefix, self.block, self.H = lens, Lq, prefix, block, H
        B, width = len(lens), max(1, -(-max(max(lens), prefix) // block))
        shared = prefix // block
        nb = shared + B * (width - shared) + spare
        perm = torch.randperm(nb, generator=g).to(torch.int32)
        own = perm[shared:shared + B * (width - shared)].view(B, width - shared)
        self.tables = torch.cat([perm[:shared].expand(B, shared), own], 1).contiguous()
        self.k, self.v = (torch.full((nb * block, H, d), float("nan"), dtype=dtype) for _ in range(2))
        self.rows = []
        for b, n in enumerate(lens):
            t = torch.arange(max(n, prefix))
            rows = self.tables[b, t // block].long() * block + t % block
            self.rows.append(rows[:n])
            fresh = rows if b == 0 else rows[prefix:]
            for x in (self.k, self.v):
                x[fresh] = torch.randn(len(fresh), H, d, generator=g).to(dtype)
        self.q = torch.randn(B, Lq, Hq, d, generator=g).to(dtype)
        self.tiers = None
        if tier_len:
            self.tiers = torch.randint(0, 3, (B, H if head_maps else 1, tier_len), generator=g, dtype=torch.uint8)
            self.tiers[torch.rand(self.tiers.shape, generator=g) < drop] = skv.DROP
            self.tiers[:, :, :prefix] = self.tiers[:1, :, :prefix]
            if not head_maps:
                self.tiers = self.tiers[:, 0]
        self.scale = d ** -0.5
        self.shape = (nb, block, H, d)

    def want(self):
        Hq = self.q.shape[2]
        parts = []
        for b, n in enumerate(self.lens):
            seen = torch.arange(n)[None, :] <= n - self.Lq + torch.arange(self.Lq)[:, None]
            seen = seen.expand(Hq, self.Lq, n).clone()
            if self.tiers is not None:
                t = self.tiers[b] if self.tiers.dim() == 3 else self.tiers[b][None].expand(self.H, -1)
                m = min(n, t.shape[1])
                seen[:, :, :m] &= (t[:, :m] != skv.DROP).repeat_interleave(Hq // self.H, 0)[:, None]
            r = self.rows[b]
            parts.append(attention(self.q[b], self.k[r], self.v[r], seen, self.scale))
        return tuple(torch.stack(x) for x in zip(*parts))

    def run(self, max_len=None, prefix=None, tables=None, lens=None, status=None, stream=None):
        q = self.q.to(DEV)
        out = torch.full_like(q, 7.0)
        lse = torch.full(q.shape[:3], 7.0, dtype=torch.float32, device=DEV)
        max_len = max(self.lens) if max_len is None else max_len
        prefix = self.prefix if prefix is None else prefix
        nb, bs, H, d = self.shape
        need = skv.attn_decode_workspace_size(len(self.lens), self.Lq, q.shape[2], H, d, max_len, prefix)
        ws = torch.empty(need, dtype=torch.uint8, device=DEV)
        skv.attn_decode(q, self.k.view(self.shape).to(DEV), self.v.view(self.shape).to(DEV),
                        (self.tables if tables is None else tables).to(DEV),
                        torch.tensor(self.lens if lens is None else lens, dtype=torch.int32, device=DEV), out, ws,
                        max_len, prefix_len=prefix, tiers=None if self.tiers is None else self.tiers.to(DEV), lse=lse,
                        dev_status=status, stream=stream)
        torch.cuda.synchronize()
        return out, lse


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16], ids=str)
@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_types_and_dimensions(d, dtype):
    for Hq, H in ((4, 2), (7, 1), (8, 8)):
        b = Batch([1, 300, 17, 64], Hq, H, d, dtype=dtype, seed=d)
        check(*b.run(), b.want(), (Hq, H, d))


@pytest.mark.parametrize("block", [1, 5, 16, 64, 300])
@pytest.mark.parametrize("Lq", [1, 3, 9])
def test_blocks_and_drafts(block, Lq):
    """A request shorter than its queries: the first ones see nothing."""
    b = Batch([Lq, 2, 513, 130], 8, 2, 64, Lq=Lq, block=block, seed=block)
    check(*b.run(), b.want(), (block, Lq))


@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("count,Lq", [(3, 1), (9, 2), (40, 4)])
def test_shared_prefix(count, Lq, d):
    lens = [448 + 7 * i for i in range(count)]
    lens[1] = 100  # ends inside the prefix
    lens[-1] = 448
    b = Batch(lens, 4, 2, d, Lq=Lq, prefix=448, seed=count)
    want = b.want()
    check(*b.run(), want, (count, Lq))
    check(*b.run(prefix=0), want, "the same without sharing") if lens[1] >= 448 else None


@pytest.mark.parametrize("head_maps", [False, True])
@pytest.mark.parametrize("drop", [0.0, 0.5, 0.97, 1.0])
def test_dropped_tokens(drop, head_maps):
    b = Batch([1500, 1024, 777], 8, 4, 128, Lq=2, prefix=512, tier_len=1200, drop=drop, head_maps=head_maps, seed=5)
    check(*b.run(), b.want(), drop)
    b = Batch([200, 40], 8, 4, 128, tier_len=300, drop=drop, head_maps=head_maps, seed=6)  # maps past the end
    check(*b.run(), b.want(), drop)


def test_long_requests_and_any_max_len():
    b = Batch([9000, 1, 2500], 4, 1, 64, seed=3)
    want = b.want()
    for max_len in (0, 100, 9000, 50000):
        check(*b.run(max_len=max_len), want, max_len)


def test_empty_requests():
    b = Batch([5, 0, 3], 4, 2, 64, seed=1)
    out, lse = b.run()
    assert (out[1] == 0).all() and (lse[1] == -float("inf")).all()
    check(out, lse, b.want())


@pytest.mark.parametrize("d", [32, 64, 128, 256])
def test_hidden_values_have_no_effect(d):
    """Infinities and NaN in dropped tokens reach nothing, in drafted tokens only the later drafts; in the prefix only
    the requests that reach them."""
    b = Batch([600, 530, 500], 4, 2, d, Lq=4, prefix=512, tier_len=520, drop=0.3, seed=d)
    for x in (b.k, b.v):
        for r, t in zip(b.rows, b.tiers):
            m = min(len(r), len(t))
            x[r[:m][t[:m] == skv.DROP]] = float("nan")
    b.v[b.rows[0][-1]], b.v[b.rows[1][-2], 0, 5] = float("nan"), float("inf")
    b.tiers[:, 505:512] = 0
    b.v[b.rows[0][506], :, 3] = float("-inf")  # past request 2's end
    for x in (b.k, b.v):
        x[b.rows[0][507:512]] = torch.where(torch.isnan(x[b.rows[0][507:512]]), 0.5, x[b.rows[0][507:512]])
        x[b.rows[0][505:506]] = 0.25
    b.k[b.rows[0][506]] = 0.25
    check(*b.run(), b.want(), d)


def test_bad_tables_and_lengths():
    b = Batch([300, 200], 4, 2, 64, seed=8)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    want = b.run(status=status)
    assert status.item() == 0
    tables = b.tables.clone()
    tables[0, 2], tables[1, 3], tables[1, 15:] = -1, b.shape[0], 1 << 30  # two in use, one behind the end
    out, lse = b.run(tables=tables, status=status)
    assert status.item() == skv.ERR_FORMAT
    cut = Batch([300, 200], 4, 2, 64, seed=8, tier_len=300)
    cut.tiers[:] = 0
    cut.tiers[0, 32:48] = cut.tiers[1, 48:64] = skv.DROP  # their tokens are left out
    check(out, lse, cut.want(), "bad entries")
    status.zero_()
    tables = b.tables.clone()
    tables[1, 13:] = 1 << 30
    out, lse = b.run(tables=tables, status=status)
    assert status.item() == 0 and torch.equal(out, want[0])
    out, lse = b.run(lens=[-5, 1 << 20], status=status)
    assert status.item() == skv.ERR_FORMAT
    assert (out[0] == 0).all()


def test_strides_and_stream():
    b = Batch([300, 40, 7], 8, 2, 128, Lq=2, tier_len=100, drop=0.5, head_maps=True, seed=4)
    want = b.want()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    check(*b.run(stream=s), want, "stream")
    q = torch.full((3, 2, 10, 136), 7.0, dtype=torch.float16, device=DEV)
    q[:, :, 1:9, :128] = b.q.to(DEV)
    out = torch.full((2, 9, 3, 128), 7.0, dtype=torch.float16, device=DEV)
    tiers = torch.zeros(3, 4, 2, 107, dtype=torch.uint8, device=DEV)[:, 1, :, 3:103]
    tiers.copy_(b.tiers.to(DEV))
    lse = torch.empty(3, 2, 8, device=DEV)
    ws = torch.empty(skv.attn_decode_workspace_size(3, 2, 8, 2, 128, 300), dtype=torch.uint8, device=DEV)
    skv.attn_decode(q[:, :, 1:9, :128], b.k.view(b.shape).to(DEV), b.v.view(b.shape).to(DEV), b.tables.to(DEV),
                    torch.tensor(b.lens, dtype=torch.int32, device=DEV), out[:, :8].permute(2, 0, 1, 3), ws, 300,
                    tiers=tiers, lse=lse)
    check(out[:, :8].permute(2, 0, 1, 3), lse, want, "strided")
    assert (out[:, 8] == 7.0).all()


def test_graph_follows_lengths_and_tables():
    """Captured once; replayed with other lengths, queries and tables, eager work between."""
    b = Batch([500, 300], 8, 2, 128, prefix=128, seed=12)
    q, k, v = b.q.to(DEV), b.k.view(b.shape).to(DEV), b.v.view(b.shape).to(DEV)
    tables, lens = b.tables.to(DEV), torch.tensor(b.lens, dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device=DEV)
    need = skv.attn_decode_workspace_size(2, 1, 8, 2, 128, 500, 128)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        skv.attn_decode(q, k, v, tables, lens, out, ws, 500, prefix_len=128, lse=lse)
    for i, now in enumerate(([500, 300], [130, 200], [499, 1])):
        lens.copy_(torch.tensor(now, dtype=torch.int32))
        q.normal_()
        if i == 1:
            tables[:, 8:] = tables[:, 8:].flip(0).clone()
        want, want_lse = torch.empty_like(out), torch.empty_like(lse)
        skv.attn_decode(q, k, v, tables, lens, want, torch.empty_like(ws), 500, prefix_len=128, lse=want_lse)
        torch.cuda.synchronize()
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        # bit for bit: the last replay's first request reads rows that hold NaN
        assert torch.equal(out.view(torch.int16), want.view(torch.int16))
        assert torch.equal(lse.view(torch.int32), want_lse.view(torch.int32))


@pytest.mark.parametrize("d,Hq,H", [(32, 4, 4), (128, 32, 8), (256, 8, 4)])
@pytest.mark.parametrize("count", [31, 35])
def test_joins_of_few_and_many_rows(count, Hq, H, d):
    """Rows joined by four waves and by one, parts of the prefix and of uneven tails."""
    lens = [640 + (900 * i) % 3001 for i in range(count)]
    b = Batch(lens, Hq, H, d, prefix=640, tier_len=2000, drop=0.6, seed=count)
    check(*b.run(), b.want(), (count, d))


def test_more_requests_than_are_cut():
    """257 requests: none is cut, the prefix still is; a long one among short ones."""
    lens = [256 + i % 3 for i in range(257)]
    lens[100], lens[256] = 1500, 0
    b = Batch(lens, 4, 4, 64, prefix=256, seed=9)
    check(*b.run(), b.want())
