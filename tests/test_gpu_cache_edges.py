"""The paged cache on the GPU where its plans, scratch, scales and waits can go wrong (reference: cache_ref.py)."""
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


# ---------------------------------------------------------------- arrays that contradict themselves
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("n", [1, 200])
def test_rows_claimed_more_than_once(dkv, fmt, n):
    """Every other of 40 sequences has all of a call's rows: an error and no outputs, instead of 20 times the work."""
    c = R.Case([(n, 300)] * 2, 2, 128, 32, fmt, seed=n)
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    bad = dkv.CacheSeqs(s.block_table[:1].repeat(40, 1), t([300] * 40), t([0] + [2 * n, 0] * 20))
    Q = torch.zeros(2, 2 * n, 128, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(Q, 3.0)
    cache.attend(Q, bad, max_rows=2 * n, out=out)
    with pytest.raises(dkv.DkvError) as e:
        cache.sync()
    assert e.value.status == 8 and bool((out == 3.0).all())
    cache.attend(Q, s, max_rows=n, out=out)
    cache.sync()
    assert not bool((out == 3.0).any())
    cache.close()


# ---------------------------------------------------------------- infinities at no weight
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("Hq,mask", [(1, dict(window=700)), (1, dict(block=128, window=640)), (3, dict(window=300, sinks=200)),
                                     (1, dict())])
def test_infinities_at_no_weight_repeat(dkv, fmt, Hq, mask):
    """Values that are not finite where the weights have fallen to 0 (keys 150 nats below the others): whatever a token
    that sees them gets, it gets every time, also where half of its unit sees less of the keys around them."""
    n, L = 512, 1500
    c = R.Case([(n, L)], 1, 128, 64, "bf16", seed=3)
    c.fmt = fmt
    g = np.random.default_rng(4)
    for j in range(L - n - 800, L, 16):
        p, sl = c.table[0, j // 64], j % 64
        c.v[p, 0, sl, g.integers(0, 128)] = [np.inf, -np.inf][j // 16 % 2] if fmt == "bf16" else np.nan
        c.k[p, 0, sl] = 0.0
        c.k[p, 0, sl, 0] = -100.0
    if fmt == "e4m3":
        quantised(c)
    Q = R.bf16(g.standard_normal((Hq, n, 128)))
    Q[:, :, 0] = 17.0                                   # -100 * 17 / sqrt(128) = -150
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    q, first = dev(Q), None
    other = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
    for i in range(60):
        if i % 3 == 1:
            other.add_(1)                               # (the pages come from HBM again, or beside other work)
        out = cache.attend(q, s, max_rows=n, **mask).view(torch.int16)
        first = out.clone() if first is None else first
        assert torch.equal(out, first), i
    cache.sync()
    cache.close()


# ---------------------------------------------------------------- waits
def test_waits_give_up(dkv):
    """On a barrier that nothing arrives on, the wait that goes by the clock gives up after 2 ms, and the wait without a clock
    (all of the chunks' roles but one) with it; the host reads the status, and the cache's attention still runs."""
    st, el = dkv.dkv_selftest_wait_timeout(2000)
    assert st == 6 and 2_000_000 <= el < 100_000_000, (st, el)
    c = R.Case([(40, 300)], 1, 128, 32, "bf16", seed=1)
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    Q = R.bf16(np.random.default_rng(0).standard_normal((2, 40, 128)))
    out = cache.attend(dev(Q), s, max_rows=40)
    cache.sync()
    R.check(out, R.attend(c, Q))
    cache.close()


# ---------------------------------------------------------------- scratch
@pytest.mark.parametrize("rows", [1, 200])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_scratch_of_infinities(dkv, rows, dtype):
    """The first attentions of a process in memory that held a mask of -infinity."""
    code = f"""
import ctypes, sys, torch
sys.path.insert(0, {str(ROOT)!r})
from paper_2608_27922_gb300 import dkv
H, d, n, rows = 2, 128, 6000, {rows}
cache = dkv.PagedCache(H, d, 64, 94, "bf16")
t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
table = torch.arange(94, dtype=torch.int32, device="cuda")[None]
torch.manual_seed(0)
K, V, Q = (torch.randn(H, n, d, device="cuda", dtype=torch.bfloat16) for _ in range(3))
cache.write(K, V, dkv.CacheSeqs(table, t([n]), t([0, n])))
seqs = dkv.CacheSeqs(table, t([n]), t([0, rows]))
Q = Q[:, :rows].contiguous()
L = dkv.lib()
size = int(L.dkv_cache_attend_scratch_size(cache.handle, 1, H, rows, rows))
scratch = torch.empty(size, dtype=torch.uint8, device="cuda")
size = scratch.numel()
got = []
for fill in (float("-inf"), float("-inf"), 0.0):
    scratch[:size // 4 * 4].view(torch.{dtype}).fill_(fill)
    out = torch.full_like(Q, 9.0)
    how = dkv.dkv_cache_attend_t(0.0, 0, 0, 1, rows)
    assert L.dkv_cache_attend(cache.handle, seqs._ref, Q.data_ptr(), H, rows, rows * d, d, out.data_ptr(), rows * d, d,
                              ctypes.byref(how), scratch.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    got.append(out)
cache.sync()
assert all(torch.equal(x, got[2]) for x in got) and not bool((got[0] == 9.0).all(-1).any())
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


# ---------------------------------------------------------------- quantised values of different magnitudes
def quantised(c):
    (c.kc, c.ks), (c.vc, c.vs) = R.quantise(c.k), R.quantise(c.v)
    c.k, c.v = R.decode(c.kc, c.ks), R.decode(c.vc, c.vs)


ROWS = [(1, 1, 1), (5, 2, 6), (40, 1, 2)]              # tokens, key heads, query heads: 8-row and 16-row units, chunks


def attend_and_check(dkv, c, Hq, Q, n):
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    out = cache.attend(dev(Q), s, max_rows=n)
    cache.sync()
    cache.close()
    R.check(out, R.attend(c, Q, rows={0, n - 1, c.rows - 1}))


@pytest.mark.parametrize("n,H,Hq", ROWS)
@pytest.mark.parametrize("size", [1.0, 0.1, 0.01, 0.001, 2.0 ** -90])
def test_zero_value_rows(dkv, n, H, Hq, size):
    """A key that most of a softmax goes to and whose value is a row of zeros (a sink): its scale byte, 127, is far above
    the other rows', and none of their weight is lost to it."""
    c = R.Case([(n, 1561), (n, 300 + n)], H, 128, 64, "bf16", seed=n)
    c.fmt = "e4m3"
    c.v *= size
    g = np.random.default_rng(7)
    Q = R.bf16(g.standard_normal((Hq, c.rows, 128)))
    for b, j in ((0, 0), (0, 777), (1, 3)):            # scores of 10 and more for all rows
        p, sl = c.table[b, j // 64], j % 64
        c.v[p, :, sl] = 0.0
        c.k[p, :, sl] = 0.0
        c.k[p, :, sl, 0] = 30.0
    Q[:, :, 0] = R.bf16(np.full(Q.shape[:2], 4.0))
    quantised(c)
    attend_and_check(dkv, c, Hq, Q, n)


@pytest.mark.parametrize("n,H,Hq", ROWS)
@pytest.mark.parametrize("top", [2.0 ** 12, 2.0 ** 30, 2.0 ** 100])
def test_large_values_in_one_column(dkv, n, H, Hq, top):
    """Rows of values that are large in one column and zero in the others: the other columns' outputs are made of small rows'
    values, whose products with their weights lie far below the large ones."""
    c = R.Case([(n, 900), (n, 2000)], H, 128, 32, "bf16", seed=n + 1)
    c.fmt = "e4m3"
    g = np.random.default_rng(8)
    big = g.random(c.v.shape[:3]) < 0.1
    c.v[big] = 0.0
    c.v[..., 77][big] = top * R.bf16(g.standard_normal(int(big.sum())))
    c.v = R.bf16(c.v)
    quantised(c)
    attend_and_check(dkv, c, Hq, R.bf16(g.standard_normal((Hq, c.rows, 128)) * 2.0), n)


@pytest.mark.parametrize("n,H,Hq", ROWS)
def test_many_small_weights(dkv, n, H, Hq):
    """A key that nearly all of a softmax goes to, with a value that is zero but in one column, and thousands of keys of weights
    around 2^-26 of its: their sum is all that the other columns hold."""
    c = R.Case([(n, 20000)], H, 128, 64, "bf16", seed=n + 2)
    c.fmt = "e4m3"
    p, sl = c.table[0, 99], 5
    c.k *= 0.25
    c.k[p, :, sl] = 0.0
    c.k[p, :, sl, 0] = 16.0
    c.v[p, :, sl] = 0.0
    c.v[p, :, sl, 3] = 1.0
    c.v = np.abs(c.v)
    quantised(c)
    Q = R.bf16(np.random.default_rng(9).standard_normal((Hq, n, 128)))
    Q[:, :, 0] = 12.75                                  # 16 * 12.75 / sqrt(128) = 18.0 = 26 log(2)
    attend_and_check(dkv, c, Hq, Q, n)


# ---------------------------------------------------------------- strides
def test_outputs_that_overlap_are_refused(dkv):
    """Rows or heads of an output that begin inside one another: no order of the writes could make them right.  Keys and
    values of a write may be one row for all."""
    H, d, n = 2, 64, 5
    c = R.Case([(n, 20)], H, d, 16, "bf16")
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    Q = torch.zeros(H, n, d, dtype=torch.bfloat16, device="cuda")
    flat = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    first = torch.zeros(1, dtype=torch.int32, device="cuda")
    for strides in ((n * d, d - 8, 1), (d - 16, H * d, 1), (8, 8, 1), (n * d, 0, 1), (0, d, 1)):
        bad = torch.as_strided(flat, (H, n, d), strides)
        for call in (lambda: cache.attend(Q, s, out=bad), lambda: cache.read(s, first, n, out=(bad, Q)),
                     lambda: cache.read(s, first, n, out=(Q, bad))):
            with pytest.raises(dkv.DkvError) as e:
                call()
            assert e.value.status == 1
    one = dev(R.bf16(np.random.default_rng(0).standard_normal((1, 1, d))))
    cache.write(one.expand(H, n, d), one.expand(H, n, d), s)
    k, v = cache.read(s, torch.full_like(first, 20 - n), n)
    cache.sync()
    assert torch.equal(k, one.expand(H, n, d)) and torch.equal(v, k)
    assert not bool(flat.any())
    cache.close()


# ---------------------------------------------------------------- cut units
@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("seqs,H,Hq,mask", [
    ([(824, 11264)], 8, 8, dict(window=2048, block=512)),            # 16, 20, 16, 16 key tiles, cut into 4 parts of 4
    ([(700, 9000)], 2, 6, dict(window=2177, sinks=5)),               # groups of 3: every unit lies differently in the tiles
    ([(900, 12000), (900, 12000)], 1, 5, dict(window=3100, block=300)),
])
def test_cut_units_longer_than_the_ends(dkv, fmt, seqs, H, Hq, mask):
    """A unit in the middle of a sequence that sees more key tiles than the first and the last one, by which units
    are cut: its last part takes the rest."""
    c = R.Case(seqs, H, 128, 64, fmt, seed=Hq)
    n = seqs[0][0]
    Q = R.bf16(np.random.default_rng(3).standard_normal((Hq, c.rows, 128)))
    cache, s = c.cache(dkv), c.device_seqs(dkv)
    out = cache.attend(dev(Q), s, max_rows=n, **mask)
    cache.sync()
    cache.close()
    R.check(out, R.attend(c, Q, heads=[0, Hq - 1], rows=set(range(0, c.rows, 9)) | {n - 1}, **mask))
