"""The paged cache on the GPU: write, read and attend against plain 64-bit arithmetic (cache_ref.py)."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def dkv():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import __graft_entry__
    __graft_entry__.build()
    from paper_2608_27922_gb300 import dkv as d
    return d


def dev(x, dtype=torch.bfloat16):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


def layout(x, how):
    """x [heads][rows][d] on the device, with other strides."""
    t = dev(x)
    H, n, d = t.shape
    if how == "rows":                                      # [rows][heads][d]
        return t.transpose(0, 1).contiguous().transpose(0, 1)
    if how == "wide":                                      # rows and heads further apart, an odd start
        w = torch.full((H, n + 2, d + 24), 9.0, dtype=t.dtype, device="cuda")
        w[:, 1:n + 1, 8:d + 8] = t
        return w[:, 1:n + 1, 8:d + 8]
    return t


def codes(cache):
    return [x if x.dtype == torch.uint8 else x.view(torch.uint8) for x in (cache.k, cache.v, cache.k_scale, cache.v_scale)]


# ---------------------------------------------------------------- write
SEQS = [
    [(1, 1)],
    [(5, 5), (0, 9), (3, 40)],
    [(70, 333), (1, 17), (130, 130), (0, 0), (16, 64)],
    [(40, 10), (2, 35)],                                   # more tokens than positions: 30 of them have none
]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("seqs", SEQS)
@pytest.mark.parametrize("H,d,page,how", [(3, 128, 16, "heads"), (2, 64, 32, "rows"), (5, 128, 128, "wide"),
                                           (1, 64, 256, "heads"), (12, 128, 64, "rows")])
def test_write_and_read(dkv, fmt, seqs, H, d, page, how):
    c = R.Case(seqs, H, d, page, fmt, seed=page + H)
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    before = [x.clone() for x in ([cache.k, cache.v] if fmt == "bf16" else codes(cache))]
    size = 2.0 ** c.rng.integers(-40, 40, (H, c.rows, 1))
    K, V = (R.bf16(c.rng.standard_normal((H, c.rows, d)) * size) for _ in range(2))
    cache.write(layout(K, how), layout(V, how), s)
    cache.sync()
    want = [x.cpu().clone() for x in before]
    for x, w, ws in ((K, want[0], want[2] if fmt == "e4m3" else None), (V, want[1], want[3] if fmt == "e4m3" else None)):
        q = R.quantise(x) if fmt == "e4m3" else None
        for b, (n, L) in enumerate(seqs):
            for i in range(n):
                j, r = L - n + i, int(c.row_start[b]) + i
                if j < 0:
                    continue
                p = int(c.table[b, j // page])
                if fmt == "e4m3":
                    w[p, :, j % page] = torch.from_numpy(q[0][:, r])
                    ws[p, :, j % page] = torch.from_numpy(q[1][:, r])
                else:
                    w[p, :, j % page] = torch.from_numpy(x[:, r]).to(torch.bfloat16)
    got = [cache.k, cache.v] if fmt == "bf16" else codes(cache)
    for g, w in zip(got, want):
        assert torch.equal(g.cpu(), w)
    # back: the new tokens' positions, two before the first one and two past the end among them
    first = c.len - np.diff(c.row_start) - 2
    k, v = layout(np.full((H, c.rows + 1, d), 7.0), how), layout(np.full((H, c.rows + 1, d), 7.0), how)
    out = cache.read(s, dev(first, torch.int32), c.rows + 1, out=(k, v))
    cache.sync()
    kd, vd = ((R.decode(a.cpu().numpy(), b.cpu().numpy()) if fmt == "e4m3" else a.double().cpu().numpy())
              for a, b in (((codes(cache)[0], codes(cache)[2]), (codes(cache)[1], codes(cache)[3])) if fmt == "e4m3"
                           else ((cache.k, None), (cache.v, None))))
    for x, pool in ((out[0], kd), (out[1], vd)):
        x = x.double().cpu().numpy()
        for b, (n, L) in enumerate(seqs):
            for i in range(n):
                j = int(first[b]) + i
                w = pool[c.table[b, j // page], :, j % page] if 0 <= j < L else np.zeros((H, d))
                assert np.array_equal(x[:, int(c.row_start[b]) + i], w), (b, i)
        assert np.all(x[:, c.rows] == 7.0)                 # behind the last sequence
    cache.close()


def test_codec_edges(dkv):
    """Rows at the edges of the scale's choice and of the codes' rounding."""
    d, rows = 128, []
    for e in (-126, -118, -111, -110, -109, -102, -101, -20, -1, 0, 7, 8, 9, 60, 127):
        for m in (1.0, 1.75, 1.7578125, 1.9921875, 1.5):   # 448 = 1.75 * 2^8 and the bf16 above it
            if e == 127 and m > 1.9921875:
                continue
            r = np.zeros(d)
            r[5] = m * 2.0 ** e
            r[6:6 + 40] = -r[5] * (1 + np.arange(40) / 128.0) * 2.0 ** -np.arange(40)   # down into the subnormal codes
            rows.append(r)
    rows.append(np.zeros(d))
    ties = np.zeros(d)
    grid = R.VALUES[:127]
    ties[:126] = (grid[1:] + grid[:-1]) / 2                # halfway between codes, exact in bf16
    ties[127] = 448
    rows.append(ties)
    rows.append(-ties)
    for bad in (math.inf, -math.inf, math.nan):
        r = np.ones(d)
        r[100] = bad
        rows.append(r)
    x = R.bf16(np.stack(rows))[None]
    c = R.Case([(x.shape[1], x.shape[1])], 1, d, 16, "e4m3")
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    cache.write(dev(x), dev(-x), s)
    k, v = cache.read(s, dev(np.zeros(1, np.int32), torch.int32), x.shape[1])
    cache.sync()
    for got, want in ((k, x), (v, -x)):
        q, sc = R.quantise(want)
        w = R.decode(q, sc)
        assert np.array_equal(got.double().cpu().numpy(), w, equal_nan=True)
        # half a step of 3 mantissa bits relative, or of the subnormal codes
        err = np.abs(w - want)[np.isfinite(want).all(-1)]
        fine = want[np.isfinite(want).all(-1)]
        step = np.ldexp(1.0, sc[np.isfinite(want).all(-1)].astype(int) - 127)[..., None]
        assert np.all(err <= np.maximum(2.0 ** -4 * np.abs(fine), 2.0 ** -10 * step))
    cache.close()


# ---------------------------------------------------------------- attend
def run(dkv, c, Hq, seed=1, how="heads", q=1.0, **kw):
    rng = np.random.default_rng(seed)
    Q = R.bf16(rng.standard_normal((Hq, c.rows, c.d)) * q)
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    out = layout(np.full((Hq, c.rows, c.d), 5.0), how)
    kw.setdefault("max_rows", max(1, max(n for n, _ in c.seqs)))
    cache.attend(layout(Q, how), s, out=out, **kw)
    cache.sync()
    kw.pop("max_rows")
    cache.close()
    return Q, out, kw


def verify(dkv, c, Hq, heads=None, rows=None, **kw):
    Q, out, kw = run(dkv, c, Hq, **kw)
    for x in ("seed", "how", "q"):
        kw.pop(x, None)
    R.check(out, R.attend(c, Q, heads=heads, rows=rows, **kw))


MASKS = [dict(), dict(block=0), dict(window=7), dict(window=40, sinks=3), dict(block=24, window=60, sinks=20),
         dict(window=1), dict(block=50, window=5), dict(window=500, sinks=130)]


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("mask", MASKS)
def test_tokens(dkv, fmt, d, mask):
    """One token each: lengths from 0 to some pages, a sequence without a token."""
    seqs = [(1, 1), (1, 0), (1, 2), (0, 30), (1, 16), (1, 31), (1, 33), (1, 64), (1, 257), (1, 700)]
    verify(dkv, R.Case(seqs, 2, d, 16, fmt, seed=3, junk=math.nan), 2, **mask)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,H,page,how", [(1, 1, 16, "heads"), (6, 2, 32, "rows"), (7, 1, 64, "wide"), (16, 2, 128, "rows"),
                                            (33, 3, 256, "heads"), (40, 2, 16, "heads"), (128, 1, 32, "rows")])
def test_groups(dkv, fmt, Hq, H, page, how):
    """Heads that share keys, in every page size and order of the tensors."""
    seqs = [(1, 90), (4, 300), (2, 2), (3, 129)]
    verify(dkv, R.Case(seqs, H, 128, page, fmt, seed=Hq, junk=math.inf), Hq, how=how, window=100, sinks=5)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("mask", MASKS)
def test_chunks(dkv, fmt, d, mask):
    """Chunks around the sizes of a tile of queries and of keys."""
    seqs = [(127, 127), (128, 400), (0, 50), (129, 129), (257, 600), (1, 300), (40, 10), (300, 301)]
    verify(dkv, R.Case(seqs, 2, d, 32, fmt, seed=11, junk=math.nan), 4, heads=[0, 3], **mask)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,H,page,how", [(3, 1, 16, "rows"), (5, 1, 64, "wide"), (14, 2, 128, "heads"), (24, 24, 256, "rows")])
def test_chunk_groups(dkv, fmt, Hq, H, page, how):
    seqs = [(200, 900), (77, 77), (333, 1500)]
    c = R.Case(seqs, H, 128, page, fmt, seed=Hq)
    rows = set(range(0, c.rows, 7)) | {199, 200, 276, 277, c.rows - 1}
    verify(dkv, c, Hq, how=how, heads=[0, Hq // 2, Hq - 1], rows=rows, window=512, sinks=64)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n,L", [(1, 20000), (1, 5003), (9, 20000), (300, 9000), (512, 12345)])
def test_long(dkv, fmt, n, L):
    """Caches that are cut into parts."""
    c = R.Case([(n, L)], 1, 128, 64, fmt, seed=L)
    verify(dkv, c, 2, rows=set(range(0, n, 37)) | {n - 1})
    verify(dkv, c, 2, rows=set(range(0, n, 37)) | {n - 1}, window=4000, sinks=700)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 20, 300])
def test_large_scores(dkv, fmt, n):
    """Scores whose maximum climbs from key to key, by far more than an exponential can hold."""
    c = R.Case([(n, 700), (n, 900)], 1, 128, 64, fmt, seed=n, keys=6.0)
    verify(dkv, c, 2, q=6.0, block=0, rows={0, n - 1, n, 2 * n - 1})
    verify(dkv, c, 2, scale=0.003, rows={0, n - 1, n, 2 * n - 1})


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_far_pages(dkv, fmt):
    """Pages whose place in the pool passes 2^31 elements: written, read and attended as near ones are."""
    H, d, page = 8, 128, 256
    n_pages = (1 << 31) // (H * page * d) + 40             # 2.2e9 elements of keys
    cache = dkv.PagedCache(H, d, page, n_pages, fmt)
    near = R.Case([(1, 700), (3, 300), (200, 500)], H, d, page, fmt, seed=9)
    small, s0 = near.cache(dkv), near.device_seqs(dkv)
    far = torch.arange(near.n_pages, device="cuda") + (n_pages - near.n_pages)
    table = torch.where(s0.block_table >= 0, s0.block_table + (n_pages - near.n_pages), s0.block_table)
    s1 = dkv.CacheSeqs(table, s0.seq_len, s0.row_start)
    g = np.random.default_rng(0)
    Q, K, V = (dev(R.bf16(g.standard_normal((H, near.rows, d)))) for _ in range(3))
    view = lambda x: x.view(torch.uint8) if x.dtype == torch.float8_e4m3fn else x
    for a, b in ((cache.k, small.k), (cache.v, small.v), (cache.k_scale, small.k_scale), (cache.v_scale, small.v_scale)):
        if a is not None:
            view(a)[far] = view(b)
    for c, s in ((small, s0), (cache, s1)):
        c.write(K, V, s)
    first = dev(near.len - np.diff(near.row_start) - 100, torch.int32)
    for a, b in zip(small.read(s0, first, near.rows), cache.read(s1, first, near.rows)):
        assert torch.equal(a, b) and bool(a.any())
    for most in (200, near.rows):
        assert torch.equal(small.attend(Q, s0, max_rows=most), cache.attend(Q, s1, max_rows=most))
    one = [dkv.CacheSeqs(s.block_table[:1].contiguous(), s.seq_len[:1].contiguous(), s.row_start[:2].contiguous())
           for s in (s0, s1)]
    assert torch.equal(small.attend(Q[:, :1], one[0], max_rows=1), cache.attend(Q[:, :1], one[1], max_rows=1))
    assert not bool(cache.k[:8].view(torch.uint8 if fmt == "e4m3" else torch.bfloat16).any())   # nothing wrapped round
    small.sync()
    cache.sync()
    cache.close()
    small.close()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_scratch_of_any_content(dkv, fmt):
    """The scratch comes uncleared: whatever it holds, also what another call left in it, the outputs keep their bits
    (single tokens and chunks that are cut into parts, in turn in the same memory)."""
    import ctypes
    L = dkv.lib()
    H, Hq, d = 2, 4, 128
    c = R.Case([(1, 9000), (200, 6000)], H, d, 64, fmt, seed=4)
    cache = c.cache(dkv)
    t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    both = c.device_seqs(dkv)
    calls = []
    for rows, start, b, n in ((1, [0, 1], 0, 1), (200, [0, 200], 1, 200), (201, [0, 1, 201], None, 200)):
        s = both if b is None else dkv.CacheSeqs(both.block_table[b:b + 1].contiguous(), both.seq_len[b:b + 1].contiguous(), t(start))
        calls.append((rows, s, n))
    Q = dev(R.bf16(np.random.default_rng(1).standard_normal((Hq, 201, d))))
    size = max(int(L.dkv_cache_attend_scratch_size(cache.handle, s.n_seq, Hq, rows, n)) for rows, s, n in calls)
    scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream

    def run(rows, s, n):
        q = Q[:, :rows].contiguous()
        out = torch.full_like(q, 9.0)
        how = dkv.dkv_cache_attend_t(0.0, 0, 0, 1, n)
        st = L.dkv_cache_attend(cache.handle, s._ref, q.data_ptr(), Hq, rows, rows * d, d, out.data_ptr(), rows * d, d,
                                ctypes.byref(how), scratch.data_ptr(), size, stream)
        assert st == 0
        return out

    want = None
    for fill in (0, 255, 1, None, None, 127):
        if fill is not None:
            scratch.fill_(fill)
        got = [run(*x) for x in calls]
        torch.cuda.synchronize()
        if want is None:
            want = got
            ref = R.attend(c, Q.double().cpu().numpy(), rows={0, 1, 100, 200})
            R.check(got[2], ref)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), fill
    cache.sync()
    cache.close()


@pytest.mark.parametrize("rows", [1, 200])
def test_scratch_of_small_integers(dkv, rows):
    """The first attention of a process, its scratch full of words that are 1 in their upper 48 or 32 bits and in their
    lower ones: a call's number and a count there would be just that, were the numbers to begin at 1."""
    code = f"""
import ctypes, sys, torch
sys.path.insert(0, {str(ROOT)!r})
from paper_2608_27922_gb300 import dkv
H, d, n, rows = 2, 128, 6000, {rows}
cache = dkv.PagedCache(H, d, 64, 94, "bf16")
t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
seqs = dkv.CacheSeqs(torch.arange(94, dtype=torch.int32, device="cuda")[None], t([n]), t([0, n]))
torch.manual_seed(0)
K, V, Q = (torch.randn(H, n, d, device="cuda", dtype=torch.bfloat16) for _ in range(3))
cache.write(K, V, seqs)
seqs = dkv.CacheSeqs(seqs.block_table, seqs.seq_len, t([0, rows]))
Q = Q[:, :rows].contiguous()
L = dkv.lib()
size = int(L.dkv_cache_attend_scratch_size(cache.handle, 1, H, rows, rows))
scratch = torch.empty(size // 8, dtype=torch.int64, device="cuda")
got = []
for fill in ((1 << (16 if rows == 1 else 32)) + 1, 0):
    scratch.fill_(fill)
    out = torch.full_like(Q, 9.0)
    how = dkv.dkv_cache_attend_t(0.0, 0, 0, 1, rows)
    assert L.dkv_cache_attend(cache.handle, seqs._ref, Q.data_ptr(), H, rows, rows * d, d, out.data_ptr(), rows * d, d,
                              ctypes.byref(how), scratch.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    got.append(out)
cache.sync()
assert torch.equal(*got) and not bool((got[0] == 9.0).all())
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


def test_whole_units_in_either_order(dkv):
    """More units than are cut, of two short sequences (round the heads) and one of more than 192 MB of keys and values
    (head by head) between them."""
    seqs = [(90, 600), (512, 9900), (33, 2000)]
    c = R.Case(seqs, 40, 128, 256, "bf16", seed=3)
    cache = c.cache(dkv)
    Q = R.bf16(np.random.default_rng(5).standard_normal((320, c.rows, 128)))
    out = cache.attend(dev(Q), c.device_seqs(dkv), max_rows=512)
    cache.sync()
    rows = {0, 31, 32, 89, 90, 91, 345, 601, 602, 634}
    R.check(out, R.attend(c, Q, heads=[0, 7, 8, 163, 319], rows=rows))
    assert bool(out.isfinite().all())
    cache.close()


@pytest.mark.parametrize("n", [1, 40])
def test_scores_of_minus_infinity(dkv, n):
    """Keys whose scores are -infinity have no weight; a token that sees no other gets zeros.  Tolerance: the weights' and
    the output's rounding to bf16, and 2^-10 for the scores (128 products and sums of 32 bits, sum |q k| scale < 40)."""
    H, d, L = 2, 128, 5000
    g = np.random.default_rng(2)
    K, V, Q = (R.bf16(g.standard_normal((H, m, d))) for m in (L, L, n))
    Q[:, :, 0] = 1.0
    t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for hidden in (3000, L):
        K[:, :hidden, 0] = -np.inf
        cache = dkv.PagedCache(H, d, 16, -(-L // 16), "bf16")
        table = torch.arange(cache.n_pages, dtype=torch.int32, device="cuda")[None]
        cache.write(dev(K), dev(V), dkv.CacheSeqs(table, t([L]), t([0, L])))
        out = cache.attend(dev(Q), dkv.CacheSeqs(table, t([L]), t([0, n])), block=0).double().cpu().numpy()
        cache.sync()
        cache.close()
        if hidden == L:
            assert not out.any()
            continue
        s = Q @ K[:, hidden:].transpose(0, 2, 1) / math.sqrt(d)
        w = np.exp(s - s.max(-1, keepdims=True))
        w /= w.sum(-1, keepdims=True)
        o, v = w @ V[:, hidden:], w @ np.abs(V[:, hidden:])
        assert (np.abs(out - o) <= v * (2.0 ** -8 + 2.0 ** -10) + 2.0 ** -8 * np.abs(o) + 1e-30).all()


@pytest.mark.parametrize("n", [1, 40])
def test_many_sequences(dkv, n):
    """More sequences than a warp's lanes, lengths of all kinds, some without tokens or positions."""
    g = np.random.default_rng(n)
    seqs = []
    for b in range(150):
        L = int(g.integers(0, 300)) if b % 7 else 0
        seqs.append((int(g.integers(0, n + 1)), L))
    c = R.Case(seqs, 1, 64, 16, "e4m3", seed=1)
    verify(dkv, c, 2, heads=[1], rows=set(range(0, c.rows, 1 + c.rows // 90)), window=100, sinks=9, max_rows=n)
    verify(dkv, c, 2, heads=[0], rows=set(range(0, c.rows, 1 + c.rows // 90)), max_rows=n)


@pytest.mark.parametrize("n", [1, 150])
@pytest.mark.parametrize("qs,ks", [(0, 0), (90, -90), (-90, 90), (-100, 60)])
def test_row_magnitudes(dkv, n, qs, ks):
    """Quantised rows and queries of very different magnitudes: scales from 2^-100 to 2^100 side by side, which
    no 16-bit product could hold as they are."""
    c = R.Case([(n, 130 + n), (n, 333)], 2, 128, 32, "e4m3", seed=n + 7)
    rng = np.random.default_rng(n)
    kb, vb = (rng.integers(-3, 3, c.ks.shape) for _ in range(2))
    vb = np.where(rng.random(c.vs.shape) < 0.3, rng.integers(-100, 100, c.vs.shape), vb)
    c.ks, c.vs = (c.ks + kb + ks).astype(np.uint8), (c.vs + vb).astype(np.uint8)
    c.k, c.v = R.decode(c.kc, c.ks), R.decode(c.vc, c.vs)
    Q = R.bf16(rng.standard_normal((4, c.rows, 128)) * 2.0 ** (qs + rng.integers(-3, 3, (4, c.rows, 1))))
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    scale = 2.0 ** -(qs + ks) / 11.0
    O = cache.attend(dev(Q), s, max_rows=n, scale=scale)
    cache.sync()
    R.check(O, R.attend(c, Q, scale=scale, rows=set(range(0, 2 * n, 11))))
    cache.close()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 5, 200])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_wild_values_stay_where_they_are_seen(dkv, fmt, n, bad):
    """A NaN or an infinity in a key or a value reaches the tokens that see it, as it would in 64 bits,
    and nobody else: tokens before it, windows past it."""
    c = R.Case([(n, 150 + n), (n, 400)], 1, 128, 16, fmt, seed=n)
    wild = [(0, 149 + n // 2, "v"), (0, 20, "v"), (1, 399 - n // 3, "v"), (1, 100, "k")]
    for b, j, which in wild:
        p, sl = c.table[b, j // 16], j % 16
        x = getattr(c, which)
        x[p, 0, sl, 3] = bad
        if fmt == "e4m3":
            x[p, 0, sl, :] = math.nan
            getattr(c, which + "c")[p, 0, sl], getattr(c, which + "s")[p, 0, sl] = 0x7F, 255
    for mask in (dict(window=90, sinks=10), dict(window=33), dict(block=0, window=250), dict(block=16, window=64, sinks=1)):
        Q, out, kw = run(dkv, c, 1, **mask)
        ref = R.attend(c, Q, **kw)
        x = out.double().cpu().numpy()
        for (h, row), (o, tol) in ref.items():
            if np.isfinite(o).all():
                assert np.isfinite(x[h, row]).all(), (mask, row)
        seen = {k: v for k, v in ref.items() if not any(
            math.isnan(t) for t in v[0]) or np.isnan(x[k]).any()}
        assert len(seen) == len(ref)                       # a NaN is not lost
        R.check(out, {k: v for k, v in ref.items() if not np.isnan(v[0]).any()})


def test_rows_behind_the_last_sequence(dkv):
    c = R.Case([(3, 50), (40, 90)], 2, 128, 16, "bf16")
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    Q = dev(np.full((2, c.rows + 9, 128), math.nan))
    Q[:, :c.rows] = 0.5
    for most in (40, 49):
        out = torch.full_like(Q, 3.0)
        cache.attend(Q, s, max_rows=most, out=out)
        cache.sync()
        assert bool((out[:, c.rows:] == 3.0).all()) and bool(torch.isfinite(out[:, :c.rows]).all())
    cache.close()


# ---------------------------------------------------------------- streams, graphs, a rollout
@pytest.mark.parametrize("n", [1, 200])
def test_graphs_and_streams(dkv, n):
    """Two captured calls of one cache replayed at once on two streams, lengths and pages changed between the
    replays; a call on a side stream."""
    c = R.Case([(n, 1000), (n, 3000)], 2, 128, 64, "e4m3", seed=5)
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    Qs = [dev(R.bf16(np.random.default_rng(i).standard_normal((4, c.rows, 128)))) for i in range(2)]
    outs, graphs = [torch.zeros_like(q) for q in Qs], [torch.cuda.CUDAGraph() for _ in Qs]
    cache.attend(Qs[0], s, max_rows=n)
    for g, q, o in zip(graphs, Qs, outs):
        with torch.cuda.graph(g):
            o.copy_(cache.attend(q, s, max_rows=n, window=900, sinks=64))
    side = [torch.cuda.Stream() for _ in Qs]
    for length in ([1000, 3000], [n, 2999], [64, 0]):
        s.seq_len.copy_(torch.tensor(length, dtype=torch.int32))
        torch.cuda.synchronize()
        for _ in range(3):
            for g, st in zip(graphs, side):
                with torch.cuda.stream(st):
                    g.replay()
        torch.cuda.synchronize()
        for q, o in zip(Qs, outs):
            want = cache.attend(q, s, max_rows=n, window=900, sinks=64)
            st = torch.cuda.Stream()
            st.wait_stream(torch.cuda.current_stream())
            other = cache.attend(q, s, max_rows=n, window=900, sinks=64, stream=st)
            torch.cuda.synchronize()
            assert torch.equal(o, want) and torch.equal(other, want)
    cache.sync()
    cache.close()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_rollout(dkv, fmt):
    """As a video goes on: each block's tokens are written, attend over [sink | window | themselves], and the
    block that leaves the window is read back and offered to the bank, whose attention reads the window from
    the cache; the pages of what nobody sees any more go to the next block."""
    H, d, N, page, frames = 2, 128, 192, 64, 5
    sink, window = 64, 2 * N                               # the block before and the block itself
    rng = np.random.default_rng(2)
    per = N // page
    n_pages = 1 + 3 * per                                  # the sink's page and three blocks
    cache = dkv.PagedCache(H, d, page, n_pages, fmt)
    bank = dkv.BankLayer(H, d, [300] * H, N)
    bank.reset()
    table = torch.full((1, frames * per), -1, dtype=torch.int32, device="cuda")
    free = list(range(n_pages))
    c = R.Case([(0, 0)], H, d, page, "bf16")
    held, allK, allV = {}, [], []
    for t in range(frames):
        for i in range(per):
            held[t * per + i] = free.pop()
            table[0, t * per + i] = held[t * per + i]
        K, V, Q = (R.bf16(rng.standard_normal((H, N, d))) for _ in range(3))
        stored = [x if fmt == "bf16" else R.decode(*R.quantise(x)) for x in (K, V)]
        allK.append(stored[0])
        allV.append(stored[1])
        L = (t + 1) * N
        s = dkv.CacheSeqs(table, torch.tensor([L], dtype=torch.int32, device="cuda"),
                          torch.tensor([0, N], dtype=torch.int32, device="cuda"))
        cache.write(dev(K), dev(V), s)
        O = cache.attend(dev(Q), s, window=window, sinks=sink, block=N, max_rows=N)
        # the reference sees every position that was ever written
        c.seqs, c.len, c.row_start, c.rows, c.page = [(N, L)], np.array([L]), np.array([0, N]), N, N
        c.table = np.arange(t + 1)[None]
        c.k, c.v = np.stack(allK), np.stack(allV)          # [blocks][H][N][d]: pages of a block each
        R.check(O, R.attend(c, Q, window=window, sinks=sink, block=N, rows=set(range(0, N, 13))))
        if t >= 1:
            k, v = cache.read(s, torch.tensor([(t - 1) * N], dtype=torch.int32, device="cuda"), N)
            assert np.array_equal(k.double().cpu().numpy(), allK[t - 1])
            assert np.array_equal(v.double().cpu().numpy(), allV[t - 1])
            bank.update(k, v, t - 1)
            kw, vw = cache.read(s, torch.tensor([t * N], dtype=torch.int32, device="cuda"), N)
            Ob = bank.attend(dev(Q), kw, vw)
            bank.sync()
            assert bool(torch.isfinite(Ob).all()) and bank.occupancy_host()[0] > 0
        for i in list(held):
            if i >= 1 and i // per <= t - 1:               # block t + 1 sees blocks t and t + 1, and the sink
                free.append(held.pop(i))
                table[0, i] = -1
    cache.sync()
    cache.close()
    bank.close()


# ---------------------------------------------------------------- refusals, inconsistent arrays
def test_refusals(dkv):
    c = R.Case([(2, 20)], 2, 128, 16, "bf16")
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    Q = dev(np.zeros((4, 2, 128)))

    def refused(status, f):
        with pytest.raises(dkv.DkvError) as e:
            f()
        assert e.value.status == status

    refused(1, lambda: cache.attend(Q, s, window=-1))
    refused(1, lambda: cache.attend(Q, s, sinks=-1))
    refused(1, lambda: cache.attend(Q, s, block=-1))
    refused(1, lambda: cache.attend(Q, s, scale=math.inf))
    refused(1, lambda: cache.attend(Q, s, max_rows=0))
    refused(1, lambda: cache.attend(Q[:1, :1].expand(4, 2, 128), s))              # one query for all heads
    refused(1, lambda: cache.attend(Q, s, out=Q[:1].expand(4, 2, 128)))
    odd = torch.zeros(4, 2, 132, dtype=torch.bfloat16, device="cuda")
    refused(1, lambda: cache.attend(odd[..., :128], s))                            # rows 264 bytes apart
    refused(1, lambda: cache.attend(torch.zeros(4 * 2 * 128 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(4, 2, 128), s))
    with pytest.raises(dkv.DkvError):
        cache.attend(Q[:3], s)                                                     # 3 query heads on 2
    with pytest.raises(ValueError):
        cache.attend(Q.float(), s)
    with pytest.raises(ValueError):
        cache.attend(Q, s, scale=-1.0)
    with pytest.raises(ValueError):
        cache.write(Q[:2], Q[:2, :1], s)
    with pytest.raises(ValueError):
        cache.read(s, torch.zeros(3, dtype=torch.int32, device="cuda"), 2)
    with pytest.raises(ValueError):
        dkv.CacheSeqs(s.block_table.long(), s.seq_len, s.row_start)
    with pytest.raises(ValueError):
        dkv.CacheSeqs(s.block_table, s.seq_len, s.row_start[:1])
    L = dkv.lib()
    import ctypes
    how = dkv.dkv_cache_attend_t(0.0, 0, 0, 1, 2)
    n = int(L.dkv_cache_attend_scratch_size(cache.handle, 1, 4, 2, 2))
    scratch = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    call = lambda p, size: L.dkv_cache_attend(cache.handle, s._ref, Q.data_ptr(), 4, 2, 256, 128, Q.data_ptr(), 256, 128,
                                              ctypes.byref(how), p, size, 0)
    assert call(scratch.data_ptr(), n - 1) == 5 and call(0, n) == 1 and call(scratch.data_ptr() + 16, n) == 1
    for bad in ((0, 128, 16, 4), (2, 96, 16, 4), (2, 128, 24, 4), (2, 128, 16, 0)):
        with pytest.raises((dkv.DkvError, RuntimeError)):
            dkv.PagedCache(*bad)
    cache.sync()                                                                   # nothing of it was enqueued
    cache.close()


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 150])
def test_inconsistent_arrays(dkv, fmt, n):
    """Pages outside the pool, lengths above the table, rows outside the tensors: an error word, and the sequences
    that are in order as they would be alone."""
    for what in ("page", "low page", "length", "negative length", "rows", "order", "chunk"):
        c = R.Case([(n, 200), (n, 300)], 2, 128, 32, fmt, seed=n)
        cache = c.cache(dkv)
        Q = R.bf16(np.random.default_rng(0).standard_normal((2, 2 * n, 128)))
        ref = R.attend(c, Q, rows=set(range(n)))
        s = c.device_seqs(dkv)
        most = n
        if what == "page":
            s.block_table[1, 5] = c.n_pages
        if what == "low page":
            s.block_table[1, 0] = -1
        if what == "length":
            s.seq_len[1] = 1 << 29
        if what == "negative length":
            s.seq_len[1] = -5
        if what == "rows":
            s.row_start[2] = 3 * n + 7
        if what == "order":
            s.row_start[2] = 0
        if what == "chunk":
            s.row_start[1:] = 2 * n                        # all rows are the first sequence's
            most = 2 * n - 1
        calls = [lambda: cache.attend(dev(Q), s, max_rows=most)]
        if what != "chunk":
            kv = dev(np.zeros((2, 2 * n, 128)))
            calls += [lambda: cache.read(s, dev(np.array([200 - n, 300 - n]), torch.int32), 2 * n), lambda: cache.write(kv, kv, s)]
        for call in calls:
            if (what == "low page" or what == "page" and n == 1) and call is not calls[0]:
                continue                                   # that page is not touched
            O = call()
            with pytest.raises(dkv.DkvError) as e:
                cache.sync()
            assert e.value.status == 8, what
            cache.sync()                                   # cleared
            if call is calls[0] and what not in ("order", "chunk"):
                R.check(O, ref)
        cache.close()
