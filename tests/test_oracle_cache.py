"""Pins of the cache oracle: the e4m3 format by its defining constants and by brute force, scales by their inequality, the
bookkeeping by its invariants (every page's count is the number of entries that map it)."""
import numpy as np
import pytest

from oracle import cache_oracle as co


def test_e4m3_constants():
    v = co.e4m3_values()
    assert v[0x7E] == 448.0 and np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and v[0x01] == 2.0 ** -9 and v[0x08] == 2.0 ** -6
    assert v[0x38] == 1.0 and v[0xB8] == -1.0 and np.all(np.diff(v[:127]) > 0)


def test_encode_is_the_nearest_value_with_ties_to_even():
    v = co.e4m3_values()[:127]
    assert np.array_equal(co.encode(v), np.arange(127)) and np.array_equal(co.encode(-v), np.arange(127) + 128)
    mid = (v[1:] + v[:-1]) / 2
    assert np.array_equal(co.encode(mid) % 2, np.zeros(126))
    x = np.random.default_rng(0).uniform(-448, 448, 4000) * 2.0 ** np.random.default_rng(1).integers(-16, 1, 4000)
    best = np.abs(np.abs(x)[:, None] - v).min(1)
    assert np.array_equal(np.abs(np.abs(co.e4m3_values()[co.encode(x)]) - np.abs(x)), best)
    assert list(co.encode([np.inf, -np.inf, np.nan]) & 127) == [127] * 3


@pytest.mark.parametrize("r", [32, 128, 160, 512])
def test_scale_is_the_least_power(r):
    x = np.random.default_rng(r).standard_normal((7, r)) * 2.0 ** np.random.default_rng(2).integers(-150, 100, (7, 1))
    x[3] = 0.0
    codes, k = co.quantize(x)
    assert k.shape == (7, -(-r // 128)) and np.all(k[3] == -126)
    for g in range(k.shape[1]):
        a = np.abs(x[:, 128 * g:128 * g + 128]).max(1)
        assert np.all(a <= 448 * 2.0 ** k[:, g]) and np.all((a > 448 * 2.0 ** (k[:, g] - 1)) | (k[:, g] == -126))
    back = co.dequantize(codes, k)
    step = np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * 2.0 ** np.repeat(k, 128, -1)[:, :r])   # half a step, or half the smallest value
    assert np.all(np.abs(back - x) <= step)


def test_bookkeeping_invariants():
    rng = np.random.default_rng(3)
    pg = co.Pages(np.full((12, 6), -1), np.zeros(25, np.int32))
    for turn in range(200):
        kind = rng.integers(4)
        n = int(rng.integers(1, 5))
        if kind == 0:
            pg.reserve(rng.integers(-1, 13, n), rng.integers(-5, 400, n))
        elif kind == 1:
            src, dst, status = pg.fork(rng.integers(-1, 13, n), rng.integers(-1, 13, n), rng.integers(-5, 400, n))
            assert all((d >= 0) == (s >= 0) for s, d in zip(src, dst))
        elif kind == 2:
            pg.free(rng.integers(-1, 13, n))
        else:
            pg.compact(int(rng.integers(0, 13)))
        ids, counts = np.unique(pg.table[pg.table >= 0], return_counts=True)
        want = np.zeros(25, np.int64)
        want[ids] = counts
        assert np.array_equal(pg.refs, want), turn
    pg.compact(25)
    used = np.flatnonzero(pg.refs > 0)
    assert np.array_equal(used, np.arange(len(used)))


def test_a_fork_continues_what_its_parent_holds():
    pg = co.Pages([[4, 1, 7, -1], [-1] * 4, [-1] * 4], [0, 1, 0, 0, 1, 0, 0, 1])
    src, dst, status = pg.fork([0, 0], [1, 2], [150, 128])
    assert status == [co.OK, co.OK] and src == [7, -1] and dst == [0, -1]
    assert pg.table.tolist() == [[4, 1, 7, -1], [4, 1, 0, -1], [4, 1, -1, -1]] and pg.refs.tolist() == [1, 3, 0, 0, 3, 0, 0, 1]
