"""Summaries of pages, the choice of pages and attention over them on the GPU."""
import numpy as np
import pytest
import torch

import cache_more_ref as ref
import cache_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dkv():
    from paper_2608_27922_gb300 import dkv
    return dkv


def t32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).cuda()


def bf(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).cuda()


def queries(case, Hq, seed=11, size=1.0):
    return cache_ref.bf16(np.random.default_rng(seed).standard_normal((Hq, case.rows, case.d)) * size)


def random_lists(case, tile, width, seed=5, most=None):
    """Ascending pages of each tile's sequence, some lists short, some empty."""
    g = np.random.default_rng(seed)
    out = np.full((case.H, case.rows // tile + len(case.seqs), width), -1, np.int32)
    for b, i, m, slot in ref.tiles(case, tile):
        pages = -(-case.seqs[b][1] // case.page)
        for h in range(case.H):
            n = min(pages, width, most if most is not None else int(g.integers(0, width + 1)))
            out[h, slot, :n] = np.sort(g.choice(pages, n, replace=False)) if n else []
    return out


# ---------------------------------------------------------------- summaries
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("page", [16, 64, 256])
def test_summaries(dkv, fmt, d, page):
    case = cache_ref.Case([(1, 1), (5, 2 * page + 3), (0, page), (page, 3 * page), (2, page - 1)], 3, d, page, fmt, seed=page)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0] * 5))
    code, scale = ref.summaries(case)
    assert np.array_equal(sums.code.cpu().numpy(), code) and np.array_equal(sums.scale.cpu().numpy(), scale)
    # the newest tokens' pages alone
    sums.code.fill_(5)
    sums.scale.fill_(6)
    c.summarise(s, sums)
    new = {(b, k) for b, (n, L) in enumerate(case.seqs) if n for k in range((L - n) // page, -(-L // page))}
    code, scale = ref.summaries(case, new, np.full_like(code, 5), np.full_like(scale, 6))
    assert np.array_equal(sums.code.cpu().numpy(), code) and np.array_equal(sums.scale.cpu().numpy(), scale)
    c.sync()


def test_summaries_at_their_limits(dkv):
    """Means on ties and at 127 2^e, tiny and large ones, sums that cancel, NaN and infinities in and behind the page."""
    case = cache_ref.Case([(1, 16 * 12 + 5)], 1, 64, 16, "bf16", seed=4, spare=1)
    k, at = case.k, case.table[0]
    g = np.random.default_rng(0)
    small = g.integers(-127, 128, (16, 64)).astype(np.float64)
    k[at[0], 0] = small                                   # means in sixteenths: ties at eighths
    k[at[1], 0] = np.where(np.arange(16)[:, None] < 8, 127, -127)
    k[at[1], 0, :, 0] = 127.0                             # the largest that 2^0 holds
    k[at[2], 0] = 2.0 ** -70
    k[at[3], 0] = 0
    k[at[4], 0] = g.standard_normal((16, 64)) * 2.0 ** 39
    k[at[5], 0, 3, 7] = np.inf
    k[at[6], 0, 15, 63] = np.nan
    k[at[7], 0] = 2.0 ** 41
    k[at[8], 0, :, 1] = np.where(np.arange(16) % 2, 1.0, -1.0) * 2.0 ** 30 + 0
    k[at[9], 0, :, 2] = [2.0 ** 60, 3.0] + [1.0] * 13 + [-2.0 ** 60]      # what is left of a sum beyond its fp32
    k[at[10], 0] = cache_ref.bf16(g.standard_normal((16, 64)) * 2.0 ** -52)
    k[at[12], 0, 5:] = np.nan                             # behind the sequence's end
    case.k = k = cache_ref.bf16(k)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0]))
    code, scale = ref.summaries(case)
    got = sums.scale.cpu().numpy()
    assert [int(got[at[i], 0]) for i in (1, 5, 6, 7)] == [127, 255, 255, 255]
    assert np.array_equal(got, scale) and np.array_equal(sums.code.cpu().numpy(), code)


# ---------------------------------------------------------------- choice
def run_choose(dkv, case, Hq, top, tile, block, sinks, local, width=None, size=1.0):
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0] * len(case.seqs)))
    Q = queries(case, Hq, size=size)
    got = c.choose(bf(Q), s, sums, top, tile=tile, block=block, sink_pages=sinks, local_pages=local, width=width)
    c.sync()
    code, scale = sums.code.cpu().numpy(), sums.scale.cpu().numpy()
    want = ref.choose(case, Q, code, scale, top, tile, block, sinks, local, got.shape[-1])
    assert np.array_equal(got.cpu().numpy(), want)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("top,tile,block,sinks,local", [(3, 1, 1, 1, 2), (0, 1, 1, 0, 1), (5, 8, 1, 2, 1), (4, 64, 0, 0, 3),
                                                        (2, 16, 20, 3, 2), (100, 3, 1, 1, 1)])
def test_choose(dkv, fmt, d, top, tile, block, sinks, local):
    case = cache_ref.Case([(3, 200), (1, 1), (40, 150), (0, 30), (20, 7), (17, 17)], 2, d, 16, fmt, seed=top)
    run_choose(dkv, case, 6, top, tile, block, sinks, local)


@pytest.mark.parametrize("H,Hq,seqs,page,top,tile", [
    (1, 1, [(1, 40000)], 16, 17, 1),             # a cluster shares 2,500 pages
    (2, 10, [(1, 9000), (1, 16), (1, 5000)], 16, 60, 1),
    (1, 128, [(1, 700)], 16, 7, 1),              # 128 query heads: two rounds of rows
    (1, 3, [(90, 1700)], 32, 9, 64),             # 192 rows
    (1, 1, [(1, 70000)], 16, 1000, 1),           # more pages than one go takes, a long list
    (1, 1, [(32, 67000)], 16, 400, 32)])         # the same for many rows
def test_choose_large(dkv, H, Hq, seqs, page, top, tile):
    case = cache_ref.Case(seqs, H, 64, page, "bf16", seed=2)
    run_choose(dkv, case, Hq, top, tile, 1, 1, 2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("H,Hq,tile", [(1, 3, 43), (2, 20, 128), (1, 9, 31), (3, 3, 128)])
def test_choose_many_rows(dkv, d, H, Hq, tile):
    """Tiles of 129, 1,280, 279 and 128 rows, and what is left of them at a sequence's end."""
    case = cache_ref.Case([(130, 2300), (7, 3900), (0, 5), (50, 60)], H, d, 16, "bf16", seed=tile)
    run_choose(dkv, case, Hq, 12, tile, 64, 1, 2)


@pytest.mark.parametrize("fmt,d,count", [("bf16", 64, 1500), ("e4m3", 128, 500), ("bf16", 128, 500), ("e4m3", 64, 500)])
def test_many_sequences(dkv, fmt, d, count):
    """Sequences of no, one or a few tokens: every tile is found, and nothing else is written."""
    g = np.random.default_rng(3)
    seqs = []
    for _ in range(count):
        n = int(g.choice([0, 1, 1, 2, 5]))
        seqs.append((n, n + int(g.integers(0, 50 if count > 1000 else 14))))
    case = cache_ref.Case(seqs, 1, d, 16, fmt, seed=7)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0] * count))
    code, scale = ref.summaries(case)
    assert np.array_equal(sums.code.cpu().numpy(), code) and np.array_equal(sums.scale.cpu().numpy(), scale)
    for tile, Hq in ((1, 2), (2, 1), (3, 9)):
        Q = queries(case, Hq)
        lists = c.choose(bf(Q), s, sums, 1, tile=tile, sink_pages=0, local_pages=1)
        want = ref.choose(case, Q, code, scale, 1, tile, 1, 0, 1, lists.shape[-1])
        assert np.array_equal(lists.cpu().numpy(), want)
        O = c.attend_chosen(bf(Q), s, lists, tile=tile)
        cache_ref.check(O, ref.attend(case, Q, want, tile))
    c.sync()


@pytest.mark.parametrize("pages,top", [(100, 28), (101, 28), (200, 56), (201, 56), (230, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_many_lists(dkv, d, pages, top):
    """480 lists of about as many pages as a CTA of a warp, of two or of eight looks at; many scores are equal."""
    g = np.random.default_rng(pages)
    seqs = [(1, int(g.integers(1, 16 * pages + 1))) for _ in range(119)] + [(1, 16 * pages)]
    case = cache_ref.Case(seqs, 4, d, 16, "bf16", seed=6)
    s, c = case.device_seqs(dkv), case.cache(dkv)
    code = g.integers(-2, 3, (case.n_pages, 4, d)).astype(np.int8)
    scale = g.integers(120, 123, (case.n_pages, 4)).astype(np.uint8)
    sums = dkv.Summaries(c, torch.from_numpy(code).cuda(), torch.from_numpy(scale).cuda())
    Q = np.round(queries(case, 12)) * 0.5
    lists = c.choose(bf(Q), s, sums, top)
    assert np.array_equal(lists.cpu().numpy(), ref.choose(case, Q, code, scale, top, 1, 1, 1, 2, lists.shape[-1]))
    c.sync()


def test_pages_given_back(dkv):
    """Pages that a window has left are neither summarised nor listed, and are no error."""
    case = cache_ref.Case([(2, 16 * 20)], 2, 64, 16, "bf16", seed=8)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    gone = [3, 4, 5, 6, 11]
    s.block_table[0, gone] = -1
    sums = dkv.Summaries(c)
    sums.code.fill_(3)
    c.summarise(s, sums, first=t32([0]))
    at = case.table[0, gone]
    assert bool((sums.code[torch.from_numpy(at).long().cuda()] == 3).all())
    code, scale = ref.summaries(case)
    scale[at] = 255
    for Hq in (2, 40):
        Q = queries(case, Hq)
        lists = c.choose(bf(Q), s, sums, 20, tile=2)
        want = ref.choose(case, Q, code, scale, 20, 2, 1, 1, 2, lists.shape[-1])
        assert np.array_equal(lists.cpu().numpy(), want) and not np.isin(want, gone).any()
        cache_ref.check(c.attend_chosen(bf(Q), s, lists, tile=2), ref.attend(case, Q, want, 2))
    c.sync()


def test_choose_ties_and_what_has_no_codes(dkv):
    """Equal pages in the order of their numbers; pages and queries that are not finite are never listed by score."""
    case = cache_ref.Case([(2, 16 * 40)], 1, 64, 16, "bf16", seed=8)
    at = case.table[0]
    for k in range(40):
        case.k[at[k]] = case.k[at[k % 3]]
    case.k[at[1], 0, 0, 0] = np.nan
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0]))
    Q = queries(case, 2)
    code, scale = ref.summaries(case)
    for which in ("plain", "zero", "nan", "huge"):
        Q2 = Q.copy()
        if which == "zero":
            Q2[:] = 0
        elif which == "nan":
            Q2[0, 0, 5] = np.nan
            Q2[1] = np.inf
        elif which == "huge":
            Q2 *= 2.0 ** 45
        got = c.choose(bf(Q2), s, sums, 5).cpu().numpy()
        assert np.array_equal(got, ref.choose(case, Q2, code, scale, 5, 1, 1, 1, 2, got.shape[-1])), which


def test_choose_strides_and_rows_behind(dkv):
    """Queries as a slice of a wider tensor and broadcast over heads; lists of slots that hold no tile are -1."""
    case = cache_ref.Case([(2, 300), (3, 400)], 2, 128, 16, "bf16", seed=8)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0, 0]))
    Q = bf(queries(case, 4))
    want = c.choose(Q, s, sums, 4, tile=2)
    wide = torch.zeros(4, 9, 3, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:7, 1] = Q
    out = torch.full_like(want, 99)
    assert torch.equal(want, c.choose(wide[:, 2:7, 1], s, sums, 4, tile=2, out=out)) and out.shape[1] == 5 // 2 + 2
    assert bool((out[:, 1] == -1).all())             # the tiles have slots 0, 2 and 3
    one = Q[:1].expand(4, 5, 128)
    assert torch.equal(c.choose(one, s, sums, 4), c.choose(one.contiguous(), s, sums, 4))


# ---------------------------------------------------------------- attention over lists
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("page", [16, 64, 256])
@pytest.mark.parametrize("Hq,H,tile,block", [(2, 2, 1, 1), (10, 2, 1, 1), (3, 1, 5, 1), (4, 4, 16, 0), (6, 2, 64, 7), (2, 1, 128, 1),
                                             (16, 1, 3, 1)])
def test_attend(dkv, fmt, d, page, Hq, H, tile, block):
    case = cache_ref.Case([(3, 500), (1, 1), (70, 290), (0, 30), (20, 7), (16, 16), (1, 1030)], H, d, page, fmt, seed=page, junk=1e30)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    lists = random_lists(case, tile, 9)
    Q = queries(case, Hq)
    O = c.attend_chosen(bf(Q), s, t32(lists), tile=tile, block=block)
    c.sync()
    cache_ref.check(O, ref.attend(case, Q, lists, tile, block))


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,H,seqs,page,tile,width", [
    (1, 1, [(1, 6000)], 64, 1, 90),              # a cluster shares a long list
    (5, 1, [(1, 4000), (1, 77)], 16, 1, 240),
    (128, 1, [(2, 600)], 16, 2, 30),               # 256 rows a tile
    (3, 3, [(300, 1200)], 128, 128, 10),
    (40, 8, [(130, 400)], 32, 64, 12),
    (2, 1, [(100, 3000), (3, 2900)], 16, 32, 180),  # clusters of four share a tile's list
    (1, 1, [(128, 1500)], 128, 128, 9),
    (1, 1, [(33, 5000)], 16, 64, 300)])             # a list longer than a CTA has threads
def test_attend_large(dkv, fmt, Hq, H, seqs, page, tile, width):
    case = cache_ref.Case(seqs, H, 128, page, fmt, seed=1)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    lists = random_lists(case, tile, width, most=width)
    Q = queries(case, Hq)
    O = c.attend_chosen(bf(Q), s, t32(lists), tile=tile)
    c.sync()
    g = np.random.default_rng(0)
    some = set(int(r) for r in g.choice(case.rows, min(case.rows, 24), replace=False)) | {0, case.rows - 1}
    want = {k: v for k, v in ref.attend(case, Q, lists, tile).items() if k[1] in some} if case.rows < 40 else \
        {k: v for k, v in ref.attend(case, Q[:, :], lists, tile).items() if k[1] in some}
    cache_ref.check(O, want)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("tile", [1, 4, 64])
def test_every_page_listed_is_dense_attention(dkv, fmt, tile):
    case = cache_ref.Case([(70, 300), (1, 200)], 2, 128, 16, fmt, seed=6)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    lists = random_lists(case, tile, 19, most=19)
    Q = queries(case, 4)
    O = c.attend_chosen(bf(Q), s, t32(lists), tile=tile)
    cache_ref.check(O, cache_ref.attend(case, Q))


@pytest.mark.parametrize("tile,pages", [(1, 7), (2, 7), (5, 7), (64, 7), (16, 7), (40, 70), (1, 70)])
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_what_is_not_finite(dkv, fmt, d, tile, pages):
    """Infinities and NaN in keys and values: they reach the rows that see them, and no others."""
    case = cache_ref.Case([(40, 16 * pages - 12)], 1, d, 16, fmt, seed=3)
    at = case.table[0][:pages]
    if fmt == "bf16":
        case.v[at[-3], 0, 2, 5], case.v[at[-2], 0, 3, 9], case.v[at[-3], 0, 9, 1] = np.inf, np.nan, -np.inf
        case.k[at[-1], 0, 1, 3] = np.nan
        case.v[at[-1], 0, 6:], case.k[at[-1], 0, 6:] = np.nan, np.inf      # behind the end
    else:
        for x, xs, full in ((case.vc, case.vs, case.v), (case.kc, case.ks, case.k)):
            for p, i in ((at[-3], 2), (at[-1], 1), (at[-1], 9)):
                x[p, 0, i], xs[p, 0, i], full[p, 0, i] = 0x7F, 255, np.nan
    else_seen = pages > 60                                            # an infinity that every row sees
    if else_seen and fmt == "bf16":
        case.v[at[2], 0, 0, 40] = np.inf
    c, s = case.cache(dkv), case.device_seqs(dkv)
    lists = random_lists(case, tile, pages, most=pages)
    Q = queries(case, 2)
    O = c.attend_chosen(bf(Q), s, t32(lists), tile=tile).double().cpu().numpy()
    want = ref.attend(case, Q, lists, tile)
    for (h, row), (o, tol) in want.items():
        fine = np.isfinite(o)
        assert not np.isfinite(O[h, row][~fine]).any(), (h, row)
        assert (np.abs(O[h, row][fine] - o[fine]) <= tol[fine]).all(), (h, row)
    assert else_seen or any(np.isfinite(o).all() for o, _ in want.values()) and any(not np.isfinite(o).all() for o, _ in want.values())


@pytest.mark.parametrize("tile", [1, 40])
def test_scores_of_minus_infinity(dkv, tile):
    """Rows all of whose scores are -infinity get zeros; large finite scores do not overflow."""
    case = cache_ref.Case([(40, 100)], 1, 64, 16, "bf16", seed=3)
    Q = np.abs(queries(case, 1)) + 1.0
    Q = cache_ref.bf16(Q)
    case.k[..., 0] = -np.inf
    c, s = case.cache(dkv), case.device_seqs(dkv)
    lists = random_lists(case, tile, 7, most=7)
    assert bool((c.attend_chosen(bf(Q), s, t32(lists), tile=tile) == 0).all())
    case = cache_ref.Case([(40, 100)], 1, 64, 16, "bf16", seed=3, keys=300.0)
    Q = queries(case, 1, size=300.0)
    O = case.cache(dkv).attend_chosen(bf(Q), case.device_seqs(dkv), t32(lists), tile=tile)
    cache_ref.check(O, ref.attend(case, Q, lists, tile))


@pytest.mark.parametrize("first", [640, 2560])
@pytest.mark.parametrize("tile", [1, 33])
def test_infinite_value_far_below_the_largest_score(dkv, tile, first):
    """A weight too small for fp32 in front of a value that is not finite: the output is not finite there, and right elsewhere."""
    case = cache_ref.Case([(33, 3300)], 1, 64, 16, "bf16", seed=3)
    for pos in range(3300):
        at = case.table[0, pos // 16], 0, pos % 16
        case.k[at] = 0.0
        case.k[at][0] = 8.0 if (pos < 640 if first == 640 else pos >= first) else -8.0
    case.v[case.table[0, 125], 0, 3, 7] = -np.inf
    case.v[case.table[0, 2], 0, 9, 20] = np.nan if first != 640 else 5.0
    c, s = case.cache(dkv), case.device_seqs(dkv)
    Q = np.zeros((1, 33, 64))
    Q[..., 0] = 40.0
    lists = np.full((1, 33 // tile + 1, 190), -1, np.int32)
    lists[0, :, :] = np.arange(190)
    O = c.attend_chosen(bf(Q), s, t32(lists), tile=tile, scale=1.0).double().cpu().numpy()
    want = ref.attend(case, Q, lists, tile, scale=1.0)
    for (h, row), (o, tol) in want.items():
        fine = np.isfinite(o)
        assert not fine.all() and not np.isfinite(O[h, row][~fine]).any()
        assert (np.abs(O[h, row][fine] - o[fine]) <= tol[fine]).all()


@pytest.mark.parametrize("tile", [1, 32])
def test_scale_strides_and_rows_behind(dkv, tile):
    case = cache_ref.Case([(33, 60), (2, 90)], 2, 128, 16, "bf16", seed=4)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    Q = queries(case, 4)
    lists = random_lists(case, tile, 6, most=6)
    extra = np.concatenate([Q, np.full((4, 3, 128), 3.0)], 1)           # rows behind the last sequence
    lists = np.concatenate([lists, np.full((2, (case.rows + 3) // tile + 2 - lists.shape[1], 6), 0, np.int32)], 1)
    wide = torch.zeros(4, 2 * (case.rows + 3), 136, dtype=torch.bfloat16, device="cuda")
    q = wide[:, ::2, :128]
    q.copy_(bf(extra))
    out = torch.full((case.rows + 3, 4, 128), 9.0, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    c.attend_chosen(q, s, t32(lists), tile=tile, scale=0.03, out=out)
    c.sync()
    cache_ref.check(out, ref.attend(case, Q, lists, tile, scale=0.03))
    assert bool((out[:, case.rows:] == 9).all())


@pytest.mark.parametrize("tile", [1, 32])
def test_faulty_lists_and_sequences(dkv, tile):
    """Entries that do not ascend, lie behind the sequence or on pages outside the pool: reported, and the other tiles are right."""
    case = cache_ref.Case([(33, 60), (2, 90)], 1, 128, 16, "bf16", seed=4, extra_cols=1)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    Q = queries(case, 2)
    good = random_lists(case, tile, 6, most=3)
    want = ref.attend(case, Q, good, tile)
    slot = [x for b, i, m, x in ref.tiles(case, tile) if b == 1][-1]
    for bad in ([3, 2, 5], [1, 1, 1], [0, 6, 7], [0, 2 ** 31 - 1, -1]):
        lists = good.copy()
        lists[0, slot, :3] = bad
        O = c.attend_chosen(bf(Q), s, t32(lists), tile=tile)
        with pytest.raises(dkv.DkvError) as e:
            c.sync()
        assert e.value.status == 8
        cache_ref.check(O, {k: v for k, v in want.items() if k[1] < 33})
    s.block_table[1, :] = 1 << 20
    O = c.attend_chosen(bf(Q), s, t32(good), tile=tile)
    with pytest.raises(dkv.DkvError):
        c.sync()
    cache_ref.check(O, {k: v for k, v in want.items() if k[1] < 33})
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0, 0]))
    c.choose(bf(Q), s, sums, 3, tile=tile)
    with pytest.raises(dkv.DkvError):
        c.sync()


@pytest.mark.parametrize("tile", [1, 32])
def test_behind_the_end_of_a_list(dkv, tile):
    """What stands behind a list's first negative entry is nothing, whatever it is."""
    case = cache_ref.Case([(33, 60), (2, 90)], 1, 128, 16, "bf16", seed=4, extra_cols=1)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    s.block_table[1, 1] = -1                       # given back
    Q = queries(case, 2)
    lists = random_lists(case, tile, 6, most=3)
    for b, i, m, slot in ref.tiles(case, tile):
        lists[0, slot, 2:] = -1
        if b == 1:
            lists[0, slot, :2] = 0, 4
    want = ref.attend(case, Q, lists, tile)
    for rest in ([2, 1, 1], [10 ** 6, 3, 2 ** 31 - 1], [1, 5, -7]):
        full = lists.copy()
        full[:, :, 3:] = rest
        cache_ref.check(c.attend_chosen(bf(Q), s, t32(full), tile=tile), want)
        c.sync()


def test_row_starts_that_go_back(dkv):
    """Arrays that contradict themselves: reported, and nothing outside the outputs is written."""
    case = cache_ref.Case([(8, 40), (8, 40), (8, 40)], 1, 64, 16, "bf16", seed=4)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    Q = bf(queries(case, 2))
    sums = dkv.Summaries(c)
    for start in ([0, 20, 4, 24], [-5, 8, 16, 24], [0, 8, 16, 10 ** 6], [24, 16, 8, 0]):
        s.row_start.copy_(t32(start))
        for tile in (1, 4, 32):
            guard = torch.full((4, 24, 64), 5.0, dtype=torch.bfloat16, device="cuda")
            c.summarise(s, sums)
            lists = c.choose(Q, s, sums, 3, tile=tile)
            c.attend_chosen(Q, s, lists, tile=tile, out=guard[1:3])
            with pytest.raises(dkv.DkvError):
                c.sync()
            assert bool((guard[0] == 5).all() and (guard[3] == 5).all())


def test_refusals(dkv):
    case = cache_ref.Case([(2, 40)], 2, 64, 16, "bf16")
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums, Q = dkv.Summaries(c), bf(queries(case, 4))
    lists = t32(np.zeros((2, 3, 4)))
    for bad in (dict(tile=129), dict(block=-1), dict(sink_pages=-1), dict(local_pages=0), dict(top=-1), dict(width=3),
                dict(width=1025), dict(top=1024)):
        kw = dict(top=2, tile=1)
        kw.update(bad)
        with pytest.raises(dkv.DkvError):
            c.choose(Q, s, sums, **kw)
    with pytest.raises(ValueError):
        c.choose(Q, s, sums, 2, tile=0)
    with pytest.raises(ValueError):
        c.choose(Q, s, sums, 2, tile=2 ** 32 + 1)
    with pytest.raises(dkv.DkvError):
        c.choose(Q[:3], s, sums, 2)
    for bad in (dict(block=-1), dict(scale=float("inf"))):
        with pytest.raises(dkv.DkvError):
            c.attend_chosen(Q, s, lists, **bad)
    with pytest.raises(dkv.DkvError):
        c.attend_chosen(Q, s, t32(np.zeros((2, 3, 1025))))
    with pytest.raises(dkv.DkvError):
        c.attend_chosen(Q, s, lists, out=torch.empty(4, 1, 64, dtype=torch.bfloat16, device="cuda").expand(4, 2, 64))
    with pytest.raises(dkv.DkvError):
        c.attend_chosen(Q, s, t32(np.zeros((2, 1, 4))), tile=129)
    for call in (lambda: c.attend_chosen(Q, s, lists, tile=2), lambda: c.attend_chosen(Q, s, lists.long()),
                 lambda: c.attend_chosen(Q, s, lists, scale=-1.0), lambda: c.attend_chosen(Q.float(), s, lists),
                 lambda: dkv.Summaries(c, code=torch.zeros(1, 2, 64, dtype=torch.int8, device="cuda")),
                 lambda: c.summarise(s, sums, first=t32([0, 0]))):
        with pytest.raises(ValueError):
            call()


def test_together_and_captured(dkv):
    """Written, summarised, chosen and attended to in one graph, replayed as a sequence grows."""
    H, d, page = 2, 128, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    case = cache_ref.Case([(1, 150), (1, 90)], H, d, page, "bf16", seed=9, extra_cols=1)
    case.table[:, -1] = [0, 0]
    c, s = case.cache(dkv), case.device_seqs(dkv)
    s.block_table[0, 10], s.block_table[1, 6] = case.n_pages - 1, case.n_pages - 2
    free = set(range(case.n_pages)) - set(case.table[0, :10].tolist()) - set(case.table[1, :6].tolist())
    a, z = sorted(free)[:2]
    s.block_table[0, 10], s.block_table[1, 6] = a, z
    case.table = s.block_table.cpu().numpy()
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0, 0]))
    Q, K, V = (torch.zeros(h, 2, d, dtype=torch.bfloat16, device="cuda") for h in (6, H, H))

    def step():
        c.write(K, V, s)
        c.summarise(s, sums)
        lists = c.choose(Q, s, sums, 3)
        return lists, c.attend_chosen(Q, s, lists)
    save = [x.clone() for x in (c.k, c.v, sums.code, sums.scale)]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lists, O = step()
    for x, y in zip((c.k, c.v, sums.code, sums.scale), save):
        x.copy_(y)
    for i in range(12):
        s.seq_len.add_(1)
        for x in (Q, K, V):
            x.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        case.k, case.v = (x.double().cpu().numpy() for x in (c.k, c.v))
        case.seqs = [(1, L) for L in s.seq_len.tolist()]
        q = Q.double().cpu().numpy()
        code, scale = sums.code.cpu().numpy(), sums.scale.cpu().numpy()
        want = ref.choose(case, q, code, scale, 3, 1, 1, 1, 2, lists.shape[-1])
        assert np.array_equal(lists.cpu().numpy(), want)
        cache_ref.check(O, ref.attend(case, q, want, 1))
    full = ref.summaries(case)
    held = np.unique(np.concatenate([case.table[0, :11], case.table[1, :7]]))
    assert np.array_equal(sums.code.cpu().numpy()[held], full[0][held])
    c.sync()


def test_two_streams(dkv):
    """Calls on two streams at once share nothing."""
    case = cache_ref.Case([(1, 5000)] * 4, 2, 128, 64, "e4m3", seed=5)
    c, s = case.cache(dkv), case.device_seqs(dkv)
    sums = dkv.Summaries(c)
    c.summarise(s, sums, first=t32([0] * 4))
    Q = [bf(queries(case, 4, seed=i)) for i in range(2)]
    want = [c.attend_chosen(q, s, c.choose(q, s, sums, 20)) for q in Q]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            lists = c.choose(Q[i], s, sums, 20, stream=streams[i])
            got[i].append(c.attend_chosen(Q[i], s, lists, stream=streams[i]))
            lists.record_stream(streams[i])
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])
