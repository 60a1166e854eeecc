"""Attention over chosen pages at its borders: scores of -infinity before values that are not finite, large and small scores, tiles
larger than a call."""
import ctypes

import numpy as np
import pytest
import torch

import cache_more_ref as ref
import cache_ref
from test_gpu_chosen import bf, queries, random_lists, t32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dkv():
    from paper_2608_27922_gb300 import dkv
    return dkv


# ---------------------------------------------------------------- scores of -infinity
WILD = {"inf": np.inf, "-inf": -np.inf, "nan": np.nan}


@pytest.mark.parametrize("wild", list(WILD))
@pytest.mark.parametrize("page", [0, 2, 97, 188])              # the first, two in the middle, one that some rows see in part
@pytest.mark.parametrize("tile", [1, 4, 33])
@pytest.mark.parametrize("run", [0, 1, 24, 110])
def test_value_behind_a_score_of_minus_infinity(dkv, wild, page, tile, run):
    """It shows, wherever the work is split: in one place among finite scores, and in a run of pages all of whose scores are
    -infinity (24: a warp's share of them, 110: a CTA's)."""
    n, L, d, col = 33, 190 * 16 - 8, 64, 21
    case = cache_ref.Case([(n, L)], 1, d, 16, "bf16", seed=3)
    pos = page * 16 + 5
    first = min(max(page - run // 2, 0), 189 - run)
    hidden = set(range(first * 16, (first + run) * 16)) | {pos}
    for p in hidden:
        case.k[case.table[0, p // 16], 0, p % 16, 0] = -np.inf
    case.v[case.table[0, page], 0, 5, col] = WILD[wild]
    Q = cache_ref.bf16(np.abs(queries(case, 1)) + 1.0)
    lists = np.full((1, n // tile + 1, 190), -1, np.int32)
    lists[0, :] = np.arange(190)
    O = case.cache(dkv).attend_chosen(bf(Q), case.device_seqs(dkv), t32(lists), tile=tile).double().cpu().numpy()
    want = ref.attend(case, Q, lists, tile, hidden=hidden)
    for (h, row), (o, tol) in want.items():
        seen = pos <= L - n + row
        assert np.isfinite(O[h, row, col]) == (not seen), (row, O[h, row, col])
        rest = np.arange(d) != col if seen else np.ones(d, bool)
        assert (np.abs(O[h, row] - o) <= tol)[rest].all(), row


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tile", [1, 40])
@pytest.mark.parametrize("pages", [7, 190])
def test_all_scores_minus_infinity(dkv, fmt, d, tile, pages):
    """Zeros, but for a value that is not finite in a place that the row sees."""
    n, L = 40, pages * 16 - 9
    case = cache_ref.Case([(n, L)], 1, d, 16, fmt, seed=3)
    Q = cache_ref.bf16(np.abs(queries(case, 1)) + 1.0)
    pos, col = (pages - 2) * 16 + 3, 13                        # some rows end before it
    at = case.table[0, pos // 16], 0, pos % 16
    if fmt == "bf16":
        case.k[..., 0] = -np.inf
        case.v[at][col] = -np.inf
        cols = [col]
    else:
        case.kc[..., 0], case.ks[:] = 0x38, 127                # ones
        case.vc[at], case.vs[at] = 0x7F, 255
        Q[..., 0] = -np.inf
        cols = list(range(d))
    lists = np.full((1, n // tile + 1, pages), -1, np.int32)
    lists[0, :] = np.arange(pages)
    O = case.cache(dkv).attend_chosen(bf(Q), case.device_seqs(dkv), t32(lists), tile=tile).double().cpu().numpy()
    for row in range(n):
        bad = cols if pos <= L - n + row else []
        assert not np.isfinite(O[0, row, bad]).any(), row
        assert (np.delete(O[0, row], bad) == 0).all(), row


# ---------------------------------------------------------------- large and small scores
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("tile", [1, 4, 33])
@pytest.mark.parametrize("top", [111, 60, 22])
def test_large_scores(dkv, fmt, d, tile, top):
    """Keys of up to 2^120 whose scores fit 32 bits: the values of the two best come out, bit for bit."""
    case = cache_ref.Case([(33, 300)], 1, d, 16, "e4m3", seed=3)
    g = np.random.default_rng(0)
    case.kc[:] = g.integers(0, 56, case.kc.shape)              # 0 .. 0.9
    case.kc[..., 1:] &= 0x0F                                   # and the others below 2^-5
    case.ks[:] = 127 + top - 1 + g.integers(0, 2, case.ks.shape)
    best = 130, 200, 261
    for i, p in enumerate(best):                               # 256 and 448 times the scale, far above the rest
        case.kc[case.table[0, p // 16], 0, p % 16, 0], case.ks[case.table[0, p // 16], 0, p % 16] = (0x78, 0x7E, 0x7E)[i], 127 + top
    case.k, case.fmt = cache_ref.decode(case.kc, case.ks), fmt
    Q = np.zeros((2, 33, d))
    Q[..., 0], Q[1, :, 1:] = 2.0, 2.0 ** -6
    lists = np.full((1, 33 // tile + 1, 19), -1, np.int32)
    lists[0, :] = np.arange(19)
    v = cache_ref.bf16(sum(case.v[case.table[0, p // 16], 0, p % 16] for p in best[1:]) / 2)
    for block in (0, 1):
        O = case.cache(dkv).attend_chosen(bf(Q[:1]), case.device_seqs(dkv), t32(lists), tile=tile, block=block, scale=0.7)
        assert np.array_equal(O[0].double().cpu().numpy(), np.broadcast_to(v, (33, d))), block
    O = case.cache(dkv).attend_chosen(bf(Q[1:]), case.device_seqs(dkv), t32(lists), tile=tile)
    assert bool(torch.isfinite(O).all())


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("tile", [1, 33])
def test_small_scale(dkv, fmt, tile):
    """Queries of zeros or far below one, a tiny scale: the mean of what a row sees."""
    case = cache_ref.Case([(33, 300)], 1, 64, 16, fmt, seed=4)
    Q = queries(case, 3)
    Q[0], Q[1] = 0, cache_ref.bf16(Q[1] * 2.0 ** -110)
    lists = random_lists(case, tile, 9)
    O = case.cache(dkv).attend_chosen(bf(Q), case.device_seqs(dkv), t32(lists), tile=tile, scale=1e-12)
    cache_ref.check(O, ref.attend(case, Q, lists, tile, scale=1e-12))


# ---------------------------------------------------------------- repetition
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,seqs,tile", [(1, [(1, 6000)], 1), (3, [(40, 900), (3, 77)], 16), (4, [(300, 3000)], 128)])
def test_same_bits_again(dkv, fmt, Hq, seqs, tile):
    case = cache_ref.Case(seqs, 1, 64, 16, fmt, seed=4)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    lists, Q = t32(random_lists(case, tile, 180)), bf(queries(case, Hq))
    want = c.attend_chosen(Q, s, lists, tile=tile)
    assert all(torch.equal(want, c.attend_chosen(Q, s, lists, tile=tile)) for _ in range(30))


# ---------------------------------------------------------------- tiles larger than the call
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,n", [(1, 1), (5, 1), (5, 2), (40, 1), (3, 5), (2, 33)])
def test_tile_larger_than_the_call(dkv, fmt, Hq, n):
    case = cache_ref.Case([(n, 700)], 1, 128, 16, fmt, seed=4)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0]))
    Q = queries(case, Hq)
    code, scale = ref.summaries(case)
    for tile in (n, n + 1, 64, 128):
        lists = c.choose(bf(Q), s, sums, 9, tile=tile)
        want = ref.choose(case, Q, code, scale, 9, tile, 1, 1, 2, lists.shape[-1])
        assert np.array_equal(lists.cpu().numpy(), want)
        cache_ref.check(c.attend_chosen(bf(Q), s, lists, tile=tile), ref.attend(case, Q, want, tile))
    c.sync()


class _Node(ctypes.Structure):
    _fields_ = [("func", ctypes.c_void_p), ("grid", ctypes.c_uint * 3), ("block", ctypes.c_uint * 3), ("shared", ctypes.c_uint),
                ("params", ctypes.c_void_p), ("extra", ctypes.c_void_p), ("kern", ctypes.c_void_p), ("ctx", ctypes.c_void_p)]


def blocks_of(call):
    """Blocks that a call's one kernel is launched with."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph(keep_graph=True)
    with torch.cuda.graph(graph):
        call()
    cu, raw, n = ctypes.CDLL("libcuda.so.1"), ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    assert cu.cuGraphGetNodes(raw, None, ctypes.byref(n)) == 0 and n.value == 1
    node, p = ctypes.c_void_p(), _Node()
    assert cu.cuGraphGetNodes(raw, ctypes.byref(node), ctypes.byref(n)) == 0
    assert cu.cuGraphKernelNodeGetParams_v2(node, ctypes.byref(p)) == 0
    return p.grid[0] * p.grid[1] * p.grid[2]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,n", [(5, 1), (40, 1), (2, 33)])
def test_blocks_of_a_tile_larger_than_the_call(dkv, fmt, Hq, n):
    """The launch goes by the tokens that a tile can have in the call."""
    case = cache_ref.Case([(n, 700)], 1, 128, 16, fmt, seed=4)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    Q = bf(queries(case, Hq))
    count = []
    for tile in (n + 1, 128):                                  # one slot either way
        lists, out = t32(random_lists(case, tile, 9)), torch.empty_like(Q)
        count.append(blocks_of(lambda: c.attend_chosen(Q, s, lists, tile=tile, out=out)))
    assert count[0] == count[1], count
