"""Norm and rotation on the GPU: dense, and on the way into the pages."""
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


def f32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()


def inputs(seed, d, pairs, rows, far=50000):
    g = np.random.default_rng(seed)
    theta = np.concatenate([10000.0 ** (-np.arange(n) / max(n, 1)) for n in pairs]).astype(np.float32).astype(np.float64)
    coord = g.integers(-far, far, (len(pairs), rows)).astype(np.int32)
    w = [(1 + 0.3 * g.standard_normal(d)).astype(np.float32).astype(np.float64) for _ in range(2)]
    return g, theta, coord, w


def bf(x):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16).cuda()


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("rows,Hq,Hk", [(1, 40, 8), (1, 1, 0), (37, 5, 1), (200, 0, 3), (33, 12, 12)])
def test_dense(dkv, d, half, norm, rows, Hq, Hk):
    pairs = [d // 2] if rows % 2 else [d // 2 - 2 * (d // 6), d // 6, d // 6]
    g, theta, coord, w = inputs(rows + d, d, pairs, rows)
    how = dkv.NormRope(d, f32(theta), axis_pairs=pairs, layout=dkv.DKV_ROPE_HALF if half else dkv.DKV_ROPE_INTERLEAVED,
                       norm=norm, eps=1e-5, q_weight=f32(w[0]), k_weight=f32(w[1]))
    eps = float(np.float32(1e-5))
    x = [cache_ref.bf16(g.standard_normal((H, rows, d)) * np.exp2(g.integers(-6, 7, (H, rows, 1)))) for H in (Hq, Hk)]
    args = [bf(a) if len(a) else None for a in x]
    out = dkv.norm_rope(*args, how, t32(coord))
    for a, y, wt in zip(x, out, w):
        if len(a):
            ref.check_rows(y, *ref.norm_rope(a, coord, theta, pairs, half, norm, eps, wt))
    # into the inputs themselves, and with rows spread out
    wide = [None if a is None else torch.zeros(a.shape[0], rows + 2, d + 16, dtype=torch.bfloat16, device="cuda")[:, 1:-1, 8:-8]
            for a in args]
    for a, z in zip(args, wide):
        if a is not None:
            z.copy_(a)
    dkv.norm_rope(*wide, how, t32(coord), out=tuple(wide))
    for y, z in zip(out, wide):
        assert y is None or torch.equal(y, z)


def test_far_positions_and_no_weights(dkv):
    """Angles of millions of radians, negative ones, and the whole range of 32 bits."""
    d, rows = 128, 6
    theta = np.concatenate([[1.0, 0.5, 3.0, 0.0], 10000.0 ** (-np.arange(60) / 60)]).astype(np.float32).astype(np.float64)
    coord = np.array([[2 ** 31 - 1, -2 ** 31, 16777217, 1000003, 0, -1]], np.int32)
    how = dkv.NormRope(d, f32(theta), norm=False)
    x = cache_ref.bf16(np.random.default_rng(1).standard_normal((2, rows, d)))
    y, none = dkv.norm_rope(bf(x), None, how, t32(coord))
    assert none is None
    ref.check_rows(y, *ref.norm_rope(x, coord, theta, [64], False, False, 0, None))
    assert torch.equal(y[:, :, 6:8], bf(x)[:, :, 6:8])                 # theta 0: bit for bit
    y, _ = dkv.norm_rope(bf(x), None, dkv.NormRope(d, f32(theta), eps=1e-6), t32(coord))
    ref.check_rows(y, *ref.norm_rope(x, coord, theta, [64], False, True, float(np.float32(1e-6)), None))


@pytest.mark.parametrize("d", [128, 64])
def test_large_eps(dkv, d):
    """An eps of the squares' own size, also where their sum passes fp32."""
    g, theta, coord, w = inputs(9, d, [d // 2], 24)
    eps = float(np.float32(1e37))
    how = dkv.NormRope(d, f32(theta), eps=eps, k_weight=f32(w[1]))
    x = cache_ref.bf16(g.standard_normal((3, 24, d)) * np.exp2(g.integers(54, 68, (3, 24, 1))))
    for x0, y, wt in zip((x, x), dkv.norm_rope(bf(x), bf(x), how, t32(coord)), (None, w[1])):
        ref.check_rows(y, *ref.norm_rope(x0, coord, theta, [d // 2], False, True, eps, wt))


@pytest.mark.parametrize("half", [False, True])
def test_extreme_rows(dkv, half):
    """Squares beyond fp32, zeros, tiny numbers, infinities and NaN, each row by itself."""
    d, rows = 64, 8
    g = np.random.default_rng(5)
    x = cache_ref.bf16(g.standard_normal((1, rows, d)))
    x[0, 0] *= 2.0 ** 120
    x[0, 1] = 0
    x[0, 2] *= 2.0 ** -100
    x[0, 3] *= 2.0 ** 62
    clean = x.copy()
    x[0, 4, 7], x[0, 5, 9], x[0, 6, 0] = np.inf, np.nan, -np.inf
    theta = (10000.0 ** (-np.arange(32) / 32)).astype(np.float32).astype(np.float64)
    coord = np.arange(rows, dtype=np.int32)[None] * 100
    how = dkv.NormRope(d, f32(theta), layout=dkv.DKV_ROPE_HALF if half else dkv.DKV_ROPE_INTERLEAVED)
    y, _ = dkv.norm_rope(bf(x), None, how, t32(coord))
    want, step = ref.norm_rope(clean, coord, theta, [32], half, True, float(np.float32(1e-6)), None)
    fine = [0, 1, 2, 3, 7]
    ref.check_rows(y[:, fine], want[:, fine], step[:, fine])
    assert torch.isnan(y[0, 4:7]).all()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("Hq,H,seqs", [(40, 8, [(1, 70), (1, 1), (1, 33), (1, 16)]), (3, 3, [(17, 40), (0, 9), (5, 5), (3, 2)]),
                                       (0, 1, [(70, 200)]), (6, 2, [(1, 1)])])
def test_into_pages(dkv, fmt, d, half, Hq, H, seqs):
    """The same as the dense call followed by a write: pages, queries, positions as coordinates; rows behind the last
    sequence are left."""
    case = cache_ref.Case(seqs, H, d, 16, "bf16", seed=3)
    page_shape = (case.n_pages, H, 16, d)
    rows, extra = case.rows, 3
    g, theta, _, w = inputs(9, d, [d // 2], rows + extra)
    pos = np.full(rows + extra, 7, np.int32)
    for b, (n, L) in enumerate(seqs):
        pos[case.row_start[b]:case.row_start[b + 1]] = np.arange(L - n, L)
    how = dkv.NormRope(d, f32(theta), layout=dkv.DKV_ROPE_HALF if half else dkv.DKV_ROPE_INTERLEAVED, q_weight=f32(w[0]), k_weight=f32(w[1]))
    K, V = (bf(g.standard_normal((H, rows + extra, d))) for _ in range(2))
    Q = bf(g.standard_normal((Hq, rows + extra, d))) if Hq else None
    caches = [dkv.PagedCache(H, d, 16, case.n_pages, fmt) for _ in range(3)]
    for c in caches:
        assert c.k.shape == page_shape
    s = case.device_seqs(dkv)
    qd, kd = dkv.norm_rope(Q, K, how, t32(pos[None]))
    caches[0].write(kd, V, s)
    out = None if Q is None else torch.full_like(Q, 7.0)
    got = caches[1].write_norm_rope(Q, K, V, s, how, out=out)
    caches[2].write_norm_rope(None, K, V, s, how, coord=t32(pos[None]))
    for c in caches[1:]:
        c.sync()
        for name in ("k", "v", "k_scale", "v_scale"):
            a, z = getattr(caches[0], name), getattr(c, name)
            assert a is None or torch.equal(a.view(torch.uint8), z.view(torch.uint8)), name
    if Hq:
        assert got is out and torch.equal(out[:, :rows], qd[:, :rows]) and bool((out[:, rows:] == 7).all())
    else:
        assert got is None


def test_faulty_sequences(dkv):
    """A page outside the pool and rows outside the call: reported, the rest as ever."""
    case = cache_ref.Case([(2, 20), (2, 40)], 2, 128, 16, "bf16", seed=1)
    case.table[1, 2] = 10 ** 6
    c = dkv.PagedCache(2, 128, 16, case.n_pages, "bf16")
    theta = f32(np.ones(64))
    K = torch.randn(2, 4, 128, device="cuda", dtype=torch.bfloat16)
    c.write_norm_rope(None, K, K, case.device_seqs(dkv), dkv.NormRope(128, theta))
    with pytest.raises(dkv.DkvError):
        c.sync()
    assert bool((c.k[int(case.table[0, 1]), :, 2:4] != 0).any())
    c.sync()


def test_refusals(dkv):
    theta = f32(np.ones(64))
    how = dkv.NormRope(128, theta)
    x = torch.zeros(2, 3, 128, device="cuda", dtype=torch.bfloat16)
    coord = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    for bad in (dict(axis_pairs=[32, 31]), dict(axis_pairs=[]), dict(axis_pairs=[70, -6]), dict(axis_pairs=[16] * 5)):
        with pytest.raises(ValueError):
            dkv.NormRope(128, theta, **bad)
    for args in ((x.float(), None), (x[..., :64], None), (None, None), (x.cpu(), None)):
        with pytest.raises(ValueError):
            dkv.norm_rope(*args, how, coord)
    with pytest.raises(ValueError):
        dkv.norm_rope(x, None, how, coord[:, :2])
    for wrong in (dict(eps=0.0), dict(eps=float("inf")), dict(layout=2)):
        with pytest.raises(dkv.DkvError):
            dkv.norm_rope(x, None, dkv.NormRope(128, theta, **wrong), coord)
    with pytest.raises(dkv.DkvError):                                  # overlapping rows of an output
        dkv.norm_rope(x, None, how, coord, out=(x[:, :1].expand(2, 3, 128), None))
    c = dkv.PagedCache(2, 128, 16, 4, "bf16")
    two = dkv.NormRope(128, theta, axis_pairs=[32, 32])
    seqs = dkv.CacheSeqs(t32([[0]]), t32([3]), t32([0, 3]))
    with pytest.raises(dkv.DkvError):                                  # positions stand for one coordinate
        c.write_norm_rope(None, x, x, seqs, two)
    with pytest.raises(ValueError):
        c.write_norm_rope(None, x, x, seqs, dkv.NormRope(64, f32(np.ones(32))))


def test_captured(dkv):
    """A captured call follows the lengths and coordinates that it finds when it is replayed."""
    case = cache_ref.Case([(1, 20), (1, 33)], 2, 128, 16, "e4m3", seed=2, extra_cols=2)
    theta = f32(10000.0 ** (-np.arange(64) / 64))
    how = dkv.NormRope(128, theta)
    c, plain = (dkv.PagedCache(2, 128, 16, case.n_pages, "e4m3") for _ in range(2))
    s = case.device_seqs(dkv)
    s.block_table[:, 3:] = 0
    Q, K, V = (torch.randn(h, 2, 128, device="cuda", dtype=torch.bfloat16) for h in (4, 2, 2))
    out = torch.empty_like(Q)
    c.write_norm_rope(Q, K, V, s, how, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.write_norm_rope(Q, K, V, s, how, out=out)
    for step in range(3):
        K.normal_()
        Q.normal_()
        s.seq_len.sub_(1)
        graph.replay()
        want = plain.write_norm_rope(Q, K, V, s, how)
        assert torch.equal(out, want)
    torch.cuda.synchronize()
    j = s.seq_len.long() - 1
    for b in range(2):
        p, q = int(s.block_table[b, int(j[b]) // 16]), int(j[b]) % 16
        assert torch.equal(c.k.view(torch.uint8)[p, :, q], plain.k.view(torch.uint8)[p, :, q])
