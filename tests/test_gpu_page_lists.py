"""The page calls on lists of no entries."""
import numpy as np
import pytest

from test_gpu_pages import Pool, dev32

pytestmark = pytest.mark.gpu


def test_empty_lists_change_nothing():
    import torch
    import paper_2410_03111_amd as L
    pool = Pool(3, 2, 9)
    pool.reserve([0, 2], [100, 64])
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    part = dev32([1, 2])[:0]
    pages = torch.arange(9 * 8, dtype=torch.int32, device="cuda").view(9, 8)
    want = pages.clone()
    for e in (none, part):
        L.copy_pages(pages, e, e)
        L.fork_sequences(pool.table, pool.refs, e, e, e, e, e, e)
        L.free_sequences(pool.table, pool.refs, e)
        L.reserve_pages(pool.table, pool.refs, e, e, e)
        L.compact_pages(pool.table, pool.refs, e, e, dev32(np.zeros(9)))        # no moves: only the map is written
    pool.same()
    assert torch.equal(pages, want)
