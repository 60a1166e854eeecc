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
