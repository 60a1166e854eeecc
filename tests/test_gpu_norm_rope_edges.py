"""Rotation without a norm of rows that are not finite."""
import numpy as np
import pytest
import torch

import cache_more_ref as ref
import cache_ref
from test_gpu_norm_rope import bf, f32, t32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("d", [64, 128])
def test_not_finite_without_norm(half, d):
    """A NaN or an infinity makes its own pair NaN or infinite; the others are as ever.  With the norm the whole row is NaN."""
    from paper_2608_27922_gb300 import dkv
    rows = 6
    x = cache_ref.bf16(np.random.default_rng(5).standard_normal((3, rows, d)))
    clean, at = x.copy(), [(0, 0, 7, np.inf), (1, 2, 9, np.nan), (2, 3, d - 1, -np.inf), (1, 5, 0, np.inf), (1, 5, d // 2 + 3, np.nan)]
    fine = np.ones(x.shape, bool)
    for h, r, e, y in at:
        x[h, r, e] = y
        clean[h, r, e] = 0
        fine[h, r, [e % (d // 2), e % (d // 2) + d // 2] if half else [e & ~1, e | 1]] = False
    theta = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32).astype(np.float64)
    coord = np.arange(rows, dtype=np.int32)[None] * 100                      # (row 0: angle 0)
    layout = dkv.DKV_ROPE_HALF if half else dkv.DKV_ROPE_INTERLEAVED
    y, _ = dkv.norm_rope(bf(x), None, dkv.NormRope(d, f32(theta), layout=layout, norm=False), t32(coord))
    got = y.double().cpu().numpy()
    assert np.array_equal(np.isfinite(got), fine)
    want, step = ref.norm_rope(clean, coord, theta, [d // 2], half, False, 0, None)
    y = torch.from_numpy(np.where(fine, got, want)).cuda()
    ref.check_rows(y, want, step)
    y, _ = dkv.norm_rope(bf(x), None, dkv.NormRope(d, f32(theta), layout=layout), t32(coord))
    got = y.double().cpu().numpy()
    assert np.array_equal(np.isnan(got).all(-1), ~fine.all(-1)) and np.array_equal(np.isfinite(got).all(-1), fine.all(-1))
