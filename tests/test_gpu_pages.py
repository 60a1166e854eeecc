"""Pages of several sequences on the GPU, against a book kept by hand: forked, grown, given back, compacted."""
import numpy as np
import pytest
import torch

import cache_more_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dkv():
    from paper_2608_27922_gb300 import dkv
    return dkv


def t32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


class Both:
    """A cache, its tables and counts on the GPU, and the book."""

    def __init__(self, dkv, n_pages, H=2, d=64, page=16, fmt="bf16", seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        shape = (n_pages, H, page, d)
        self.dkv, self.page = dkv, page
        byte = lambda s: torch.randint(0, 120, s, generator=g, device="cuda", dtype=torch.uint8)
        if fmt == "e4m3":
            k, v = (byte(shape).view(torch.float8_e4m3fn) for _ in range(2))
            self.cache = dkv.PagedCache(H, d, page, n_pages, fmt, k=k, v=v, k_scale=byte(shape[:3]) + 100, v_scale=byte(shape[:3]) + 90)
        else:
            k, v = (torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
            self.cache = dkv.PagedCache(H, d, page, n_pages, fmt, k=k, v=v)
        self.refs = self.cache.new_refs()
        self.book = ref.Book(n_pages, page, [x.cpu().numpy() for x in self.pools()])
        self.table = None

    def pools(self):
        c = self.cache
        out = [c.k.view(torch.uint8).view(*c.k.shape[:3], -1), c.v.view(torch.uint8).view(*c.v.shape[:3], -1)]
        return out if c.k_scale is None else out + [c.k_scale, c.v_scale]

    def start(self, lengths, cols):
        n = len(lengths)
        self.table = self.dkv.PageTable(torch.full((n, cols), -1, dtype=torch.int32, device="cuda"), t32([0] * n))
        self.book.table, self.book.length = [[] for _ in range(n)], [0] * n
        self.extend(lengths)

    def extend(self, add, fits=True):
        self.cache.extend(self.refs, self.table, t32(add))
        assert self.book.extend(add) == fits
        if fits:
            self.cache.sync()
        else:
            with pytest.raises(self.dkv.DkvError) as e:
                self.cache.sync()
            assert e.value.status == 5
        self.check()

    def other(self, n, cols):
        junk = torch.randint(-5, 1 << 20, (n, cols), dtype=torch.int32, device="cuda")
        return self.dkv.PageTable(junk, t32([77] * n))

    def fork(self, parents, cols=None):
        to = self.other(len(parents), cols or self.table.block_table.shape[1])
        self.cache.fork(self.refs, self.table, t32(parents), to)
        self.book.fork(parents)
        self.table = to
        self.cache.sync()
        self.check()

    def release(self, first, last):
        self.cache.release(self.refs, self.table, t32(first), t32(last))
        self.book.release(first, last)
        self.cache.sync()
        self.check()

    def compact(self, keep, cols=None):
        to = self.other(len(keep), cols or self.table.block_table.shape[1])
        start = np.concatenate([[0], np.cumsum([len(k) for k in keep])])
        flat = np.concatenate([np.asarray(k, np.int32) for k in keep] + [np.zeros(0, np.int32)])
        self.cache.compact(self.refs, self.table, t32(flat), t32(start), to)
        self.book.compact(keep)
        self.table = to
        self.cache.sync()
        self.check()

    def check(self):
        t = self.table
        assert t.seq_len.tolist() == self.book.length
        assert np.array_equal(t.block_table.cpu().numpy(), self.book.padded(t.block_table.shape[1]))
        assert self.refs.tolist() == self.book.refs
        for a, z in zip(self.pools(), self.book.rows):
            assert np.array_equal(a.cpu().numpy(), z)


@pytest.mark.parametrize("fmt,d,page,H", [("bf16", 64, 16, 2), ("e4m3", 128, 32, 3), ("bf16", 128, 256, 1), ("e4m3", 64, 256, 2)])
def test_a_life(dkv, fmt, d, page, H):
    """Lengths of zero, one, whole and ragged pages; forks of forks, growth of shared and own pages, windows, ends."""
    x = Both(dkv, 90, H, d, page, fmt)
    x.start([0, 1, page, page + 1, 3 * page - 1], cols=8)
    x.extend([0, 0, 0, 0, 0])
    x.fork([4, 4, 3, -1, 1, 1, 1, 0])
    x.extend([1, 1, 2, 3, page - 1, page, 0, 1])          # shared: two both in the call; one of three stays out
    x.extend([0, page, 1, 0, 1, 1, 1, 0])
    x.fork([0, 1, 2, 3, 4, 5, 6, 7, 6, 1], cols=9)
    x.release([page, 0, 0, 0, 2, 0, 1, 5, 0, 2 * page],
              [2 * page, 0, 2 ** 31 - 1, page, 2 ** 31 - 1, 2 ** 31 - 1, page, 1, -3, 2 ** 31 - 1])
    x.extend([1, page + 3, 4, 0, 1, 2, 0, 1, 1, 1])
    x.compact([[j for j in range(n) if j < page or j >= 2 * page or b != 0] for b, n in enumerate(x.book.length)])
    lens = list(x.book.length)
    x.compact([list(range(n)) if b % 2 else list(range(n))[::-1] for b, n in enumerate(lens)], cols=11)
    x.compact([[0] * 3 + list(range(0, n, 2)) if n else [] for n in x.book.length])
    x.fork([-1] * 2)
    assert x.refs.sum() == 0
    x.extend([2 * page, 1])
    assert x.table.block_table[:, :2].tolist() == [[0, 1], [2, -1]]


@pytest.mark.parametrize("seed", range(6))
def test_at_random(dkv, seed):
    g = np.random.default_rng(seed)
    page = int(g.choice([16, 32]))
    x = Both(dkv, int(g.integers(60, 9000)), 1, 64, page, str(g.choice(["bf16", "e4m3"])), seed)
    x.start(g.integers(0, 4 * page, 5).tolist(), cols=16)
    for _ in range(14):
        n, what = len(x.book.length), g.integers(4)
        lens = x.book.length
        holes = any(p < 0 for row in x.book.table for p in row)
        if what == 0:
            x.fork(g.integers(-1, n, int(g.integers(1, 9))).tolist())
        elif what == 1:
            add = [int(min(g.integers(0, 40), 16 * page - m)) for m in lens]
            try:
                need_ok = sum(-(-(m + a) // page) + 1 for m, a in zip(lens, add)) < len(x.book.free())
            except ValueError:
                need_ok = False
            if need_ok and not any(m % page and row[m // page] < 0 for m, row in zip(lens, x.book.table)):
                x.extend(add)
        elif what == 2:
            lo = [int(g.integers(0, m + 2)) for m in lens]
            x.release(lo, [int(a + g.integers(0, 3 * page)) if g.random() < 0.6 else 2 ** 31 - 1 for a in lo])
        elif not holes and sum(-(-m // page) for m in lens) < len(x.book.free()):
            x.compact([sorted(g.choice(m, int(g.integers(0, m + 1)), replace=False).tolist()) if m else [] for m in lens])


def test_many_sequences(dkv):
    """4,096 sequences on one shared page; all grow but every seventh; then all end."""
    x = Both(dkv, 9001, 1, 64, 16, "bf16")
    x.start([21], cols=3)
    x.fork([0] * 4096)
    x.extend([0 if b % 7 == 3 else 1 + b % 13 for b in range(4096)])
    x.fork(list(range(4095, -1, -1)))
    x.extend([b % 3 for b in range(4096)])
    x.release([0] * 4096, [2 ** 31 - 1] * 4096)
    assert x.refs.sum() == 0


def test_last_holder_keeps_the_page(dkv):
    x = Both(dkv, 20)
    x.start([5], cols=2)
    x.fork([0, 0, 0])
    x.extend([1, 1, 1])
    assert x.table.block_table[:, 0].tolist() == [1, 2, 0] and x.refs[:4].tolist() == [1, 1, 1, 0]


def test_too_few_pages(dkv):
    """Nothing changes, and the next call works."""
    x = Both(dkv, 6)
    x.start([40, 20], cols=6)
    x.extend([30, 30], fits=False)
    x.fork([0, 0, 1])
    x.extend([1, 1, 13], fits=False)
    x.extend([1, 0, 0])
    with pytest.raises(dkv.DkvError):
        to = x.other(3, 6)
        before = to.block_table.clone()
        keep = list(range(1, 41)) + list(range(40)) + list(range(20))
        x.cache.compact(x.refs, x.table, t32(keep), t32([0, 40, 80, 100]), to)
        x.cache.sync()
    assert torch.equal(before, to.block_table) and to.seq_len.tolist() == [77] * 3
    x.check()


@pytest.mark.parametrize("what", ["page", "free", "length", "negative", "full", "occupied"])
def test_faults_change_nothing(dkv, what):
    """extend and compact on arrays that contradict themselves."""
    x = Both(dkv, 40)
    x.start([40, 20, 7], cols=4)
    add, keep, start = [1, 2, 3], [1, 2, 3, 0], [0, 2, 3, 4]
    t = x.table
    if what == "page":
        t.block_table[1, 1] = 40
    elif what == "free":
        x.refs[int(t.block_table[1, 1])] = 0
    elif what == "length":
        t.seq_len[1] = 65
    elif what == "negative":
        add, keep = [1, -1, 3], [1, -1, 3, 0]
    elif what == "full":
        add, keep = [30, 1, 1], [40, 2, 3, 0]
    else:
        t.block_table[1, 2] = 9
        x.refs[9] = 1
        add, start = [1, 20, 1], [0, 2, 1, 4]
    save = t.block_table.clone(), t.seq_len.clone(), x.refs.clone(), [p.clone() for p in x.pools()]
    to = x.other(3, 4)
    kept = to.block_table.clone()
    for call in (lambda: x.cache.extend(x.refs, t, t32(add)),
                 lambda: x.cache.compact(x.refs, t, t32(keep), t32(start), to)):
        call()
        with pytest.raises(dkv.DkvError) as e:
            x.cache.sync()
        assert e.value.status == 8
        assert torch.equal(t.block_table, save[0]) and torch.equal(t.seq_len, save[1]) and torch.equal(x.refs, save[2])
        assert all(torch.equal(a, z) for a, z in zip(x.pools(), save[3])) and torch.equal(to.block_table, kept)


def test_faults_of_fork_and_release(dkv):
    """Parents outside the table, pages outside the pool, pages given up twice."""
    x = Both(dkv, 40)
    x.start([40, 20, 7], cols=4)
    x.table.block_table[1, 1] = 4000
    to = x.other(4, 4)
    x.cache.fork(x.refs, x.table, t32([1, 3, -2, 0]), to)
    with pytest.raises(dkv.DkvError):
        x.cache.sync()
    assert to.seq_len.tolist() == [20, 0, 0, 40] and to.block_table[:, 1].tolist() == [-1, -1, -1, 1]
    assert int(x.refs.min()) >= 0
    x.refs.zero_()
    x.cache.release(x.refs, to, t32([0] * 4), t32([100] * 4))
    with pytest.raises(dkv.DkvError):
        x.cache.sync()
    assert int(x.refs.abs().max()) == 0


def test_refusals(dkv):
    x = Both(dkv, 8)
    x.start([3, 3], cols=2)
    c, refs, t = x.cache, x.refs, x.table
    with pytest.raises(dkv.DkvError):
        c.fork(refs, t, t32([0, 1]), t)                   # the same table
    with pytest.raises(dkv.DkvError):
        c.fork(refs, t, t32([0, 1]), dkv.PageTable(torch.zeros(2, 1, dtype=torch.int32, device="cuda"), t32([0, 0])))
    with pytest.raises(dkv.DkvError):
        c.compact(refs, t, t32([0]), t32([0, 0, 1]), x.other(3, 2))
    with pytest.raises(dkv.DkvError):
        c.extend(torch.zeros(9, dtype=torch.int32, device="cuda")[1:], t, t32([0, 0]))     # not 16-byte aligned
    for call in (lambda: c.extend(refs[:4], t, t32([0, 0])), lambda: c.extend(refs, t, t32([0])),
                 lambda: c.release(refs, t, t32([0]), t32([0, 0])), lambda: c.fork(refs, t, t32([0]), t),
                 lambda: c.compact(refs, t, t32([0]), t32([0, 1]), x.other(2, 2)),
                 lambda: dkv.PageTable(t.block_table.long(), t.seq_len), lambda: dkv.PageTable(t.block_table.cpu(), t.seq_len)):
        with pytest.raises(ValueError):
            call()


def test_captured(dkv):
    """A step of forks and growth in a graph, replayed on what the last one left."""
    x = Both(dkv, 60)
    x.start([5, 20, 33], cols=6)
    a, z = x.table, x.other(3, 6)
    parent, add = t32([0, 1, 2]), t32([0, 0, 0])

    def step():
        x.cache.fork(x.refs, a, parent, z)
        x.cache.extend(x.refs, z, add)
        a.block_table.copy_(z.block_table)
        a.seq_len.copy_(z.seq_len)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for p, m in (([1, 1, 0], [3, 1, 20]), ([0, 0, 0], [1, 1, 1]), ([2, -1, 1], [0, 30, 16])):
        parent.copy_(t32(p))
        add.copy_(t32(m))
        graph.replay()
        torch.cuda.synchronize()
        x.book.fork(p)
        assert x.book.extend(m)
        x.check()
    x.cache.sync()


def test_next_to_write_and_attend(dkv):
    """Two continuations of one prompt: grown, written and attended to as two sequences that share nothing would be."""
    H, d, page = 2, 128, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    rnd = lambda n: torch.randn(H, n, d, generator=g, device="cuda", dtype=torch.bfloat16)
    c, plain = dkv.PagedCache(H, d, page, 20, "bf16"), dkv.PagedCache(H, d, page, 20, "bf16")
    refs = c.new_refs()
    prompt = dkv.PageTable(torch.full((1, 4), -1, dtype=torch.int32, device="cuda"), t32([0]))
    c.extend(refs, prompt, t32([21]))
    K, V = rnd(21), rnd(21)
    c.write(K, V, dkv.CacheSeqs(prompt.block_table, prompt.seq_len, t32([0, 21])))
    two = dkv.PageTable(torch.zeros(2, 4, dtype=torch.int32, device="cuda"), t32([0, 0]))
    c.fork(refs, prompt, t32([0, 0]), two)
    c.extend(refs, two, t32([2, 2]))
    k2, v2, q2 = rnd(4), rnd(4), rnd(4)
    rows = t32([0, 2, 4])
    s = dkv.CacheSeqs(two.block_table, two.seq_len, rows)
    c.write(k2, v2, s)
    p = dkv.CacheSeqs(t32([[4, 9], [2, 7]]), t32([21, 21]), t32([0, 21, 42]))
    plain.write(torch.cat([K, K], 1), torch.cat([V, V], 1), p)
    p = dkv.CacheSeqs(p.block_table, t32([23, 23]), rows)
    plain.write(k2, v2, p)
    assert torch.equal(c.attend(q2, s, max_rows=2), plain.attend(q2, p, max_rows=2))
    c.sync()
    assert int(refs.sum()) == 4 and int((refs == 2).sum()) == 1
