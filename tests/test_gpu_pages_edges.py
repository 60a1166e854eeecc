"""Pages of several sequences: counts that contradict the tables, streams other than the current one, choices after a move."""
import numpy as np
import pytest
import torch

import cache_more_ref as ref
import cache_ref
from test_gpu_chosen import bf, queries
from test_gpu_pages import Both, t32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dkv():
    from paper_2608_27922_gb300 import dkv
    return dkv


@pytest.mark.parametrize("held", [1, 2])
def test_compact_of_a_page_named_more_often_than_counted(dkv, held):
    """Reported, and no count goes below zero."""
    x = Both(dkv, 40)
    x.start([40, 40, 40], cols=4)
    t = x.table
    t.block_table[1, 0] = t.block_table[2, 0] = t.block_table[0, 0]
    x.refs[int(t.block_table[0, 0])] = held
    to = x.other(3, 4)
    x.cache.compact(x.refs, t, t32([1, 2, 3]), t32([0, 1, 2, 3]), to)
    with pytest.raises(dkv.DkvError) as e:
        x.cache.sync()
    assert e.value.status == 8 and int(x.refs.min()) == 0
    x.cache.release(x.refs, to, t32([0] * 3), t32([9] * 3))
    x.cache.sync()
    assert int(x.refs.min()) == 0


def test_streams_other_than_the_current_one(dkv):
    """Each call's work and scratch belong to the stream that it is given, a torch stream or a raw handle."""
    x = Both(dkv, 60, fmt="e4m3")
    x.start([5, 20, 33], cols=6)
    side = torch.cuda.Stream()
    for handle in (side, side.cuda_stream):
        n = len(x.book.length)
        add, parents = t32([3] * n), [1, 1, 0, 2][:n + 1]
        keep = [list(range(0, m + 3, 2)) for m in (x.book.length[p] for p in parents)]
        start = np.concatenate([[0], np.cumsum([len(k) for k in keep])])
        args = t32(parents), t32(np.concatenate(keep)), t32(start), t32([10] * len(parents)), t32([2 ** 31 - 1] * len(parents))
        forked, kept = x.other(len(parents), 6), x.other(len(parents), 6)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        x.cache.extend(x.refs, x.table, add, stream=handle)
        x.cache.fork(x.refs, x.table, args[0], forked, stream=handle)
        x.cache.compact(x.refs, forked, args[1], args[2], kept, stream=handle)
        x.cache.release(x.refs, kept, args[3], args[4], stream=handle)
        junk = [torch.full((1 << 16,), 0x7F, dtype=torch.uint8, device="cuda") for _ in range(8)]    # (not the calls' scratch)
        x.book.extend([3] * n)
        x.book.fork(parents)
        x.book.compact(keep)
        x.book.release([10] * len(parents), [2 ** 31 - 1] * len(parents))
        x.table = kept
        side.synchronize()
        x.check()
        assert all(bool((j == 0x7F).all()) for j in junk)
    x.cache.sync()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_choice_after_a_move(dkv, fmt):
    """Compacted sequences, whose moved pages are summarised anew, and one that ends earlier, whose last page is: choices and
    attention as of the positions that they hold now."""
    H, d, page = 2, 64, 16
    x = Both(dkv, 90, H, d, page, "bf16")
    c = x.cache
    if fmt == "e4m3":
        c = x.cache = dkv.PagedCache(H, d, page, 90, "e4m3")
        x.refs = c.new_refs()
        x.book = ref.Book(90, page, [p.cpu().numpy() for p in x.pools()])
    x.start([300, 211], cols=24)
    seqs = dkv.CacheSeqs(x.table.block_table, x.table.seq_len, t32([0, 300, 511]))
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    K, V = (torch.randn(H, 511, d, generator=g, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    c.write(K, V, seqs)
    x.book.rows = [p.cpu().numpy() for p in x.pools()]
    sums = dkv.Summaries(c)
    c.summarise(seqs, sums)
    n = [3, 2]

    def look(first):
        case = cache_ref.Case([(a, L) for a, L in zip(n, x.book.length)], H, d, page, "bf16")
        case.table, case.n_pages = x.table.block_table.cpu().numpy(), 90
        k, v = (p.cpu().numpy() for p in x.pools()[:2])
        if fmt == "e4m3":
            case.k, case.v = (cache_ref.decode(a, s.cpu().numpy()) for a, s in zip((k, v), x.pools()[2:]))
        else:
            case.k, case.v = c.k.double().cpu().numpy(), c.v.double().cpu().numpy()
        s = dkv.CacheSeqs(x.table.block_table, x.table.seq_len, t32(case.row_start))
        c.summarise(s, sums, first=t32(first))
        Q = queries(case, 4)
        lists = c.choose(bf(Q), s, sums, 4, tile=2)
        want = ref.choose(case, Q, *ref.summaries(case), 4, 2, 1, 1, 2, lists.shape[-1])
        assert np.array_equal(lists.cpu().numpy(), want)
        cache_ref.check(c.attend_chosen(bf(Q), s, lists, tile=2), ref.attend(case, Q, want, 2))
        c.sync()
    look([0, 0])
    x.compact([[j for j in range(300) if j < 40 or j % 3], list(range(30, 211))])
    look([0, 0])
    x.release([203, 100], [2 ** 31 - 1] * 2)
    look([length - 1 for length in x.book.length])
