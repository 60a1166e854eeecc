"""The paged cache on the GPU where its plans, scratch, scales and waits can go wrong (reference: cache_ref.py)."""
import numpy as np
import pytest
import torch

import cache_ref as R

pytestmark = pytest.mark.gpu


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
