"""The oracle's counts where a fork takes a row that still maps pages behind its first entry."""
import numpy as np

from oracle import cache_oracle as co


def counts(pages):
    ids = pages.table[(pages.table >= 0) & (pages.table < len(pages.refs))]
    return np.bincount(ids, minlength=len(pages.refs))


def test_oracle_a_fork_releases_what_the_rest_of_the_childs_row_maps():
    pg = co.Pages([[-1, 1, 2, -1], [-1] * 4], [0, 1, 1, 0, 0])
    assert pg.fork([0], [1], [130])[2] == [co.OK]
    assert pg.fork([0], [1], [130])[2] == [co.OK]       # the child's first entry maps nothing: taken again
    assert np.array_equal(pg.refs, counts(pg))
    pg.free([0, 1])
    assert not pg.refs.any() and np.all(pg.table == -1)


def test_oracle_random_forks_of_rows_without_a_first_page():
    rng = np.random.default_rng(0)
    table = np.full((9, 5), -1)
    table[:5, 1:] = np.arange(20).reshape(5, 4)
    pg = co.Pages(table, np.where(np.arange(40) < 20, 1, 0))
    for _ in range(100):
        n = int(rng.integers(1, 5))
        pg.fork(list(rng.integers(-1, 9, n)), list(rng.integers(-1, 9, n)), list(rng.integers(0, 321, n)))
        assert np.array_equal(pg.refs, counts(pg))
        if rng.random() < 0.2:
            pg.free(rng.integers(0, 9, 2))
            row = int(rng.integers(0, 9))
            pg.reserve([row], [320])
            if pg.maps(pg.table[row, 0]):       # its first page is dropped, as behind a window
                pg.refs[pg.table[row, 0]] -= 1
                pg.table[row, 0] = -1
