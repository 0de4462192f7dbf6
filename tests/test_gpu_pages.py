"""Page operators against plain numpy: reserve, fork, compact, free and copy,
with tables, counts, lengths and every row of the pool compared exactly."""
import numpy as np
import pytest
import torch

from paper_2606_08635_amd import skv

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Pool:
    """A pool on the host with the operators' definitions, and its copy on the GPU."""

    def __init__(self, L, blocks, block, H, d, seed=0):
        self.rng = np.random.default_rng(seed)
        self.block = block
        self.k, self.v = (self.rng.integers(0, 1 << 15, (L, blocks, block, H, d)).astype(np.uint16) for _ in range(2))
        self.refs = np.zeros(blocks, np.int32)

    def cdiv(self, n):
        return -(-n // self.block)

    def take(self, n):
        free = np.flatnonzero(self.refs == 0)[:n]
        assert len(free) == n
        self.refs[free] = 1
        return free

    def requests(self, lens, width):
        """Tables of new requests on scattered pages."""
        tables = np.full((len(lens), width), -7, np.int32)
        free = self.rng.permutation(np.flatnonzero(self.refs == 0))
        at = 0
        for b, n in enumerate(lens):
            m = self.cdiv(n)
            tables[b, :m] = free[at:at + m]
            at += m
            self.refs[tables[b, :m]] = 1
        return tables

    def upload(self):
        up = lambda x: torch.from_numpy(x.view(np.int16)).to(DEV).view(torch.float16)  # noqa: E731
        self.dk, self.dv, self.drefs = up(self.k), up(self.v), torch.from_numpy(self.refs).to(DEV)

    def check(self):
        torch.cuda.synchronize()
        assert np.array_equal(self.drefs.cpu().numpy(), self.refs)
        assert np.array_equal(self.dk.cpu().numpy().view(np.uint16), self.k)
        assert np.array_equal(self.dv.cpu().numpy().view(np.uint16), self.v)

    def rows(self, table, n):
        t = np.arange(n)
        return table[t // self.block], t % self.block

    def build(self, table, tokens, shared, out):
        """`out` becomes the table of `tokens` (indexes into `table`), its first `shared` pages table's own."""
        m = self.cdiv(len(tokens))
        out[:shared] = table[:shared]
        np.add.at(self.refs, table[:shared], 1)
        out[shared:m] = self.take(m - shared)
        src, dst = self.rows(table, len(table) * self.block), self.rows(out, len(tokens))
        move = slice(shared * self.block, None)
        for x in (self.k, self.v):
            x[:, dst[0][move], dst[1][move]] = x[:, src[0][tokens[move]], src[1][tokens[move]]]


def dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x, dtype)).to(DEV)


def status():
    return torch.full((1,), -1, dtype=torch.int32, device=DEV)


def workspace(rows, blocks, tokens):
    return torch.full((skv.pages_workspace_size(rows, blocks, tokens),), 0xA5, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("block", [1, 5, 16, 300])
def test_fork_reserve_free(block):
    p = Pool(2, 400 if block < 300 else 40, block, 2, 32, seed=block)
    lens = [33, 0, 5 * block, 1] if block > 1 else [33, 0, 17, 1]
    width = p.cdiv(max(lens)) + 2
    tables = p.requests(lens, width)
    p.upload()
    parents = [0, 3, 0, 2, 1, 0, 2]
    out = np.full((len(parents), width + 1), -9, np.int32)
    d_out, d_lens, st, ws = dev(out), dev(np.full(len(parents), -9)), status(), workspace(len(parents), len(p.refs), width * block + block)
    skv.pages_fork(p.dk, p.dv, p.drefs, dev(tables), dev(lens), dev(parents), d_out, d_lens, ws, st)
    for c, b in enumerate(parents):
        p.build(tables[b], np.arange(lens[b]), lens[b] // block, out[c])
    p.check()
    child = np.array([lens[b] for b in parents])
    assert st.item() == 0 and np.array_equal(d_out.cpu().numpy(), out) and d_lens.cpu().tolist() == child.tolist()
    # room for more tokens, none for one child; one keeps its length
    grown = np.minimum(child + np.array([1, block, 2 * block, 0, 3, 1, -1]), (width + 1) * block)
    grown = np.maximum(grown, 0)
    skv.pages_reserve(p.drefs, d_out, dev(child), dev(grown), block, ws, st)
    for c in range(len(parents)):
        a, b = p.cdiv(child[c]), p.cdiv(grown[c])
        out[c, a:max(a, b)] = p.take(max(0, b - a))
    p.check()
    assert st.item() == 0 and np.array_equal(d_out.cpu().numpy(), out)
    end = np.maximum(child, grown)
    skv.pages_free(p.drefs, d_out, dev(end), block, st)
    for c in range(len(parents)):
        np.subtract.at(p.refs, out[c, :p.cdiv(end[c])], 1)
    p.check()
    assert st.item() == 0


@pytest.mark.parametrize("block,drop", [(1, 0.5), (5, 0.3), (16, 0.0), (16, 0.4), (16, 1.0), (300, 0.5)])
def test_compact(block, drop):
    p = Pool(3, 1200 if block < 300 else 40, block, 2, 32, seed=block)
    lens = [700, 0, 257, 256, 1, 90]
    if block == 1:
        lens = [300, 0, 129, 1]
    width = p.cdiv(max(lens))
    tables = p.requests(lens, width)
    tier_len = 600
    tiers = p.rng.integers(0, 3, (len(lens), tier_len)).astype(np.uint8)
    tiers[p.rng.random(tiers.shape) < drop] = skv.DROP
    tiers[0, :2 * block] = 0  # full pages before the first dropped token
    p.upload()
    out = np.full((len(lens), width), -9, np.int32)
    d_out, d_lens, st = dev(out), dev(np.full(len(lens), -9)), status()
    skv.pages_compact(p.dk, p.dv, p.drefs, dev(tables), dev(lens), dev(tiers, np.uint8), d_out, d_lens,
                      workspace(len(lens), len(p.refs), width * block), st)
    kept = []
    for b, n in enumerate(lens):
        m = min(n, tier_len)
        keep = np.concatenate([tiers[b, :m] != skv.DROP, np.ones(n - m, bool)])
        tokens = np.flatnonzero(keep)
        first = n if keep.all() else int(np.argmin(keep))
        p.build(tables[b], tokens, first // block, out[b])
        kept.append(len(tokens))
    p.check()
    assert st.item() == 0 and np.array_equal(d_out.cpu().numpy(), out) and d_lens.cpu().tolist() == kept


def test_wide_rows_and_many_requests():
    """More requests than one scan covers, a pool of several scan rounds, rows of 4 KB."""
    p = Pool(1, 40000, 2, 1, 32, seed=3)
    lens = p.rng.integers(0, 12, 2500)
    tables = p.requests(lens, 6)
    p.upload()
    out, parents = np.full((2600, 7), -9, np.int32), p.rng.integers(0, 2500, 2600)
    d_out, d_lens, st, ws = dev(out), dev(np.zeros(2600)), status(), workspace(2600, 40000, 14)
    skv.pages_fork(p.dk, p.dv, p.drefs, dev(tables), dev(lens), dev(parents), d_out, d_lens, ws, st)
    for c, b in enumerate(parents):
        p.build(tables[b], np.arange(lens[b]), lens[b] // 2, out[c])
    p.check()
    assert st.item() == 0 and np.array_equal(d_out.cpu().numpy(), out)
    skv.pages_free(p.drefs, d_out, d_lens, 2, st)
    for c, b in enumerate(parents):
        np.subtract.at(p.refs, out[c, :p.cdiv(lens[b])], 1)
    p.check()
    p = Pool(2, 30, 16, 16, 128, seed=4)
    tables = p.requests([200], 13)
    p.upload()
    out = np.full((1, 13), -9, np.int32)
    tiers = (np.arange(200) % 3 == 1)[None] * skv.DROP
    d_out, st = dev(out), status()
    skv.pages_compact(p.dk, p.dv, p.drefs, dev(tables), dev([200]), dev(tiers, np.uint8), d_out, dev([0]), workspace(1, 30, 208), st)
    p.build(tables[0], np.flatnonzero(tiers[0] == 0), 0, out[0])
    p.check()
    assert st.item() == 0 and np.array_equal(d_out.cpu().numpy(), out)


@pytest.mark.parametrize("shape", [(3, 16, 2, 64), (1, 1, 1, 32), (2, 300, 8, 128)])
def test_copy(shape):
    L, block, H, d = shape
    a, b = Pool(L, 20, block, H, d, seed=1), Pool(L, 33, block, H, d, seed=2)
    a.upload(), b.upload()
    src, dst = a.rng.integers(0, 20, 12), a.rng.permutation(33)[:12]  # a source may be used twice
    st = status()
    skv.pages_copy(a.dk, a.dv, b.dk, b.dv, dev(src), dev(dst), st)
    b.k[:, dst], b.v[:, dst] = a.k[:, src], a.v[:, src]
    a.check(), b.check()
    assert st.item() == 0
    skv.pages_copy(b.dk, b.dv, b.dk, b.dv, dev([0]), dev([1]), st)  # inside one pool
    b.k[:, 1], b.v[:, 1] = b.k[:, 0], b.v[:, 0]
    b.check()


def test_refused_calls_change_nothing():
    p = Pool(1, 12, 4, 1, 32, seed=5)
    tables = p.requests([9, 4], 4)  # 3 + 1 pages
    p.upload()
    d_out, d_lens, st, ws = dev(np.full((3, 4), -9)), dev([-9, -9, -9]), status(), workspace(16, 12, 16)
    t = dev(tables)

    def fork(parents, lens=(9, 4), tab=t, out=None):
        n = len(parents)
        skv.pages_fork(p.dk, p.dv, p.drefs, tab, dev(lens), dev(parents), (d_out if out is None else out)[:n].contiguous(),
                       d_lens[:n], ws, st)
        p.check()
        assert d_lens.cpu().tolist() == [-9, -9, -9]
        return st.item()

    assert fork([0, 2]) == skv.ERR_FORMAT  # no such parent
    assert fork([0, -1]) == skv.ERR_FORMAT
    assert fork([0], lens=(17, 4)) == skv.ERR_FORMAT  # longer than its table
    assert fork([1], lens=(9, -1)) == skv.ERR_FORMAT
    assert fork([1], lens=(9, 5)) == skv.ERR_FORMAT  # an entry that holds no page
    other = tables.copy()
    other[0, 1] = np.flatnonzero(p.refs == 0)[0]
    assert fork([0], tab=dev(other)) == skv.ERR_FORMAT  # a free page
    assert fork([0], out=dev(np.full((1, 2), -9))) == skv.ERR_CAPACITY  # too narrow
    wide = dev(np.full((9, 4), -9))
    skv.pages_fork(p.dk, p.dv, p.drefs, t, dev([9, 4]), dev([0] * 9), wide, dev([0] * 9), ws, st)
    p.check()
    assert st.item() == skv.ERR_CAPACITY and (wide == -9).all()  # 9 new pages, 8 free
    assert (d_out == -9).all()
    new = t.clone()
    skv.pages_reserve(p.drefs, new, dev([9, 4]), dev([16, 17]), 4, ws, st)
    assert st.item() == skv.ERR_FORMAT
    p.check()
    q = Pool(1, 5, 4, 1, 32)
    tab = q.requests([9, 4], 4)
    q.upload()
    new = dev(tab)
    skv.pages_reserve(q.drefs, new, dev([9, 4]), dev([13, 8]), 4, workspace(2, 5, 16), st)
    q.check()
    assert st.item() == skv.ERR_CAPACITY and torch.equal(new, dev(tab))
    skv.pages_copy(p.dk, p.dv, p.dk, p.dv, dev([0, 12]), dev([1, 2]), st)
    p.check()
    assert st.item() == skv.ERR_FORMAT
    tiers = torch.zeros(2, 9, dtype=torch.uint8, device=DEV)
    skv.pages_compact(p.dk, p.dv, p.drefs, dev(other), dev([9, 4]), tiers, d_out[:2].contiguous(), d_lens[:2], ws, st)
    p.check()
    assert st.item() == skv.ERR_FORMAT


def test_free_passes_over_what_is_not_held():
    p = Pool(1, 12, 4, 1, 32, seed=6)
    tables = p.requests([9, 4, 8], 3)
    p.upload()
    bad = tables.copy()
    bad[1, 0] = 12
    st = status()
    skv.pages_free(p.drefs, dev(bad), dev([9, 4, 8]), 4, st)
    p.refs[tables[0, :3]] -= 1
    p.refs[tables[2, :2]] -= 1
    p.check()
    assert st.item() == skv.ERR_FORMAT
    skv.pages_free(p.drefs, dev(tables), dev([9, 4, 13]), 4, st)  # twice; a bad length
    p.refs[tables[1, 0]] -= 1
    p.check()
    assert st.item() == skv.ERR_FORMAT and (p.refs == 0).all()


def test_free_without_entries():
    """Tables of no width: requests of no tokens hold nothing, a longer one is reported."""
    refs, st = torch.ones(8, dtype=torch.int32, device=DEV), torch.full((2,), -1, dtype=torch.int32, device=DEV)
    tables = torch.zeros(3, 0, dtype=torch.int32, device=DEV)
    skv.pages_free(refs, tables, torch.zeros(3, dtype=torch.int32, device=DEV), 16, st[:1])
    skv.pages_free(refs, tables, torch.tensor([0, 5, 0], dtype=torch.int32, device=DEV), 16, st[1:])
    assert st.tolist() == [skv.OK, skv.ERR_FORMAT] and (refs == 1).all()
