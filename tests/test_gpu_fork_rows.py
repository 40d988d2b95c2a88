"""Forks onto rows whose first entry maps nothing while later ones do."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from test_gpu_pages import Pool

pytestmark = pytest.mark.gpu


def counts(pool):
    t = pool.table.cpu().numpy()
    return np.bincount(t[(t >= 0) & (t < len(pool.o.refs))], minlength=len(pool.o.refs))


# a table that a plan changes itself, one whose rows take a launch of their own, lists beyond a plan's LDS
@pytest.mark.parametrize("n_seqs, max_pages, n_pages, forks", [(6, 4, 40, 2), (40, 300, 20000, 30), (2500, 5, 9000, 1100)])
def test_forks_onto_rows_whose_first_entry_maps_nothing(n_seqs, max_pages, n_pages, forks):
    rng = np.random.default_rng(n_seqs)
    table = np.full((n_seqs, max_pages), -1)
    rows = n_seqs // 2
    table[:rows, 1:] = rng.permutation(n_pages)[:rows * (max_pages - 1)].reshape(rows, -1)
    pool = Pool(n_seqs, max_pages, n_pages, table, np.isin(np.arange(n_pages), table).astype(np.int32))
    for _ in range(3):
        pair = rng.permutation(n_seqs)
        status = pool.fork(np.resize(pair[forks:], forks), pair[:forks], rng.integers(0, 64 * max_pages + 1, forks))[2]
        assert co.OK in status
        assert np.array_equal(pool.refs.cpu().numpy(), counts(pool))
    pool.free(list(range(n_seqs)))
    assert int(pool.refs.abs().sum()) == 0
