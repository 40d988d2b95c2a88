"""Latents into 8-bit pages against the oracle, byte for byte: every rank form, ranges that begin and end inside a page, special values,
bytes that are not the call's to write, unmapped pages, single tokens against whole prompts."""
import numpy as np
import pytest

import lorc_inputs as gen
from lorc_testlib import PAGE, page_gather_indices
from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu


def layer(r_k, r_v):
    import paper_2410_03111_amd as L
    n = max(r_k, r_v)
    n_kv = max(1, -(-n // 128))
    return L.layer_desc(256, n_kv, n_kv, 128, r_k, r_v, 1e4)


def run(values, r_k, r_v, begins, ends, max_tokens=None, table=None, table_q8=None, n_pages=None, fill=0xA5):
    """values [n_pages, 64, r_k + r_v] bf16 bits.  Returns (got pool, expected pool)."""
    import torch
    import paper_2410_03111_amd as L
    d = layer(r_k, r_v)
    idx = page_gather_indices(r_k, r_v)
    n_pages = len(values)
    pool = np.zeros((n_pages, PAGE * (r_k + r_v)), np.uint16)
    for p in range(n_pages):
        pool[p][idx] = values[p]
    table_q8 = table[::-1].copy() if table_q8 is None else table_q8
    size = L.page_bytes_quantized(d)
    got = torch.full((n_pages, size), fill, dtype=torch.uint8, device="cuda")
    i32 = lambda v: torch.as_tensor(np.ascontiguousarray(v, np.int32)).cuda()  # noqa: E731
    cap = max(max(e - b for b, e in zip(begins, ends)), 0) if max_tokens is None else max_tokens
    L.quantize_latents(d, torch.from_numpy(pool.view(np.uint8)).cuda(), i32(table), i32(begins), i32(ends), cap, got, i32(table_q8))
    want = np.full((n_pages, size), fill, np.uint8)
    for s, (b, e) in enumerate(zip(begins, ends)):
        b = max(b, 0)
        for t in range(b, min(e, b + cap)):
            if t // PAGE >= table.shape[1] or t // PAGE >= table_q8.shape[1]:
                continue
            src, dst, slot = table[s, t // PAGE], table_q8[s, t // PAGE], t % PAGE
            if not (0 <= src < n_pages and 0 <= dst < n_pages):
                continue
            x = gen.bf16_to_f32(values[src, slot]).astype(np.float64)
            for part, cols in ((False, slice(0, r_k)), (True, slice(r_k, r_k + r_v))):
                codes, k = co.quantize(x[cols])
                want[dst][idx[slot][cols]] = codes
                for g in range(len(k)):
                    want[dst, co.scale_index(r_k, r_v, slot, 128 * g, part)] = k[g] + 127
    return got.cpu().numpy(), want


def latents(n_pages, r, seed, spread=8):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((n_pages, PAGE, r)) * 2.0 ** rng.integers(-spread, spread + 1, (n_pages, PAGE, 1)) * np.arange(1, r + 1) ** -0.7
    return gen.bf16_bits(x.astype(np.float32))


def ids(b, max_pages, seed=0):
    return np.random.default_rng(seed).permutation(b * max_pages).reshape(b, max_pages).astype(np.int32)


@pytest.mark.parametrize("r_k, r_v", [(32, 32), (64, 96), (128, 128), (160, 288), (512, 512), (576, 32), (1024, 1024), (32, 1120)])
def test_prompts(r_k, r_v):
    table = ids(3, 3)
    got, want = run(latents(9, r_k + r_v, r_k), r_k, r_v, [0, 0, 0], [192, 65, 1], table=table)
    assert np.array_equal(got, want)


@pytest.mark.parametrize("begins, ends", [([5, 63, 64, 100], [6, 64, 65, 101]), ([0, 30, 63, 127], [64, 34, 130, 129]), ([10, 0, 50, 191], [10, 0, 20, 192]),
                                          ([7, 8, 17, 33], [15, 16, 31, 170]), ([-9, 190, 0, 1], [3, 400, 5, 250])])
def test_ranges(begins, ends):
    table = ids(4, 3, 1)
    got, want = run(latents(12, 160 + 64, 3), 160, 64, begins, ends, table=table)
    assert np.array_equal(got, want)


def test_longer_ranges_are_cut_off():
    table = ids(2, 4, 2)
    got, want = run(latents(8, 64 + 32, 4), 64, 32, [3, 60], [200, 130], max_tokens=70, table=table)
    assert np.array_equal(got, want)


def test_ranges_at_the_ends_of_int32():
    table = ids(4, 3, 6)
    got, want = run(latents(12, 64 + 32, 7), 64, 32, [5, 2 ** 31 - 1, -2 ** 31, 3], [-2 ** 31, 2 ** 31 - 1, 2, 2 ** 31 - 1], max_tokens=250, table=table)
    assert np.array_equal(got, want)


def test_no_rows_behind_the_last_sequence_and_refused_arguments():
    import torch
    import paper_2410_03111_amd as L
    d = layer(64, 32)
    size, size_q8 = L.page_bytes(d), L.page_bytes_quantized(d)
    cache, got = torch.zeros(4 * size, dtype=torch.uint8, device="cuda"), torch.full((4 * size_q8,), 9, dtype=torch.uint8, device="cuda")
    table = torch.tensor([[0], [1], [2]], dtype=torch.int32, device="cuda")
    begin, end = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((2,), 64, dtype=torch.int32, device="cuda")
    L.quantize_latents(d, cache, table, begin, end, 64, got, table)                 # a table of three rows, two sequences
    assert not bool((got[:2 * size_q8] == 9).any()) and bool((got[2 * size_q8:] == 9).all())
    good = dict(cache=cache, block_table=table, pos_begin=begin, pos_end=end, max_tokens=64, cache_q8=got, block_table_q8=table)
    for key, value, error in (("cache", cache.cpu(), TypeError), ("cache", cache.to(torch.int16), TypeError), ("cache_q8", got[::2], TypeError),
                              ("block_table", table.to(torch.int64), TypeError), ("block_table", table[:1], ValueError),
                              ("block_table_q8", table[:1], ValueError), ("pos_end", end[:1], ValueError), ("pos_begin", [0, 0], TypeError),
                              ("max_tokens", -1, L.LorcError), ("cache", cache[:100], L.LorcError), ("cache_q8", got[8:], L.LorcError)):
        with pytest.raises(error):
            L.quantize_latents(d, **{**good, key: value})


def test_unmapped_pages_and_tables_of_different_width():
    table, table_q8 = ids(2, 3, 3), ids(2, 3, 4)[:, :2].copy()
    table[0, 1], table_q8[1, 0] = -1, 6
    got, want = run(latents(6, 64 + 32, 5), 64, 32, [0, 0], [192, 192], table=table, table_q8=table_q8)
    assert np.array_equal(got, want)


def test_special_values():
    r = 128 + 64
    x = gen.bf16_to_f32(latents(2, r, 6, spread=0)).copy()
    x[0, 0] = 0.0                                            # nothing but zeros
    x[0, 1, 3] = np.inf
    x[0, 2, 130], x[0, 2, 140] = -np.inf, np.nan
    x[0, 3] = np.nan                                         # nothing finite
    x[0, 4] = 448.0                                          # the largest code, at every scale
    x[0, 5] = 450.0                                          # one bf16 step above: the next power
    x[0, 6] = 2.0 ** -130                                    # below the least scale's codes
    x[0, 7] = 3.3e38
    x[0, 8] *= 1e-38
    x[0, 9, ::2] = -0.0
    x[0, 10, :] = 2.0 ** -133 * np.arange(r)                 # subnormal bf16
    x[0, 11, :] = 17.0 * 2.0 ** np.repeat(np.arange(24), 8)  # (and midpoints between codes)
    x[0, 12] = 1.0 + np.arange(r) / 128
    table = np.array([[0], [1]], np.int32)
    with np.errstate(all="ignore"):
        got, want = run(gen.bf16_bits(x.astype(np.float32)), 128, 64, [0, 0], [64, 20], table=table, table_q8=np.array([[1], [0]], np.int32))
    idx = page_gather_indices(128, 64)
    nan = (want[1][idx] & 127) == 127
    assert np.array_equal((got[1][idx] & 127) == 127, nan)   # (a NaN's sign is not defined)
    got[1][idx[nan]] = want[1][idx[nan]] = 127
    assert np.array_equal(got, want)


def test_token_by_token_is_the_same_as_at_once():
    import torch
    import paper_2410_03111_amd as L
    d = layer(288, 64)
    values = latents(3, 288 + 64, 7)
    pool = np.zeros((3, PAGE * 352), np.uint16)
    for p in range(3):
        pool[p][page_gather_indices(288, 64)] = values[p]
    i32 = lambda v: torch.as_tensor(np.ascontiguousarray(v, np.int32)).cuda()  # noqa: E731
    cache, table = torch.from_numpy(pool.view(np.uint8)).cuda(), i32([[2, 0, 1]])
    pools = [torch.zeros(3, L.page_bytes_quantized(d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    L.quantize_latents(d, cache, table, i32([0]), i32([150]), 150, pools[0], table)
    for t in range(150):
        L.quantize_latents(d, cache, table, i32([t]), i32([t + 1]), 1, pools[1], table)
    assert torch.equal(*pools)


def test_pools_beyond_4_gib():
    import torch
    import paper_2410_03111_amd as L
    d = layer(1024, 1024)
    n = 40000                                                # 262144-byte pages: 10 GiB, 8-bit 5 GiB
    cache = torch.zeros(n, L.page_bytes(d) // 2, dtype=torch.bfloat16, device="cuda")
    cache[n - 1] = 3.0
    cache[n - 2] = torch.randn(cache.shape[1], device="cuda")
    out = torch.zeros(n, L.page_bytes_quantized(d), dtype=torch.uint8, device="cuda")
    i32 = lambda v: torch.as_tensor(np.ascontiguousarray(v, np.int32)).cuda()  # noqa: E731
    L.quantize_latents(d, cache.view(torch.uint8), i32([[n - 1, n - 2]]), i32([0]), i32([128]), 128, out, i32([[n - 3, n - 1]]))
    small = torch.zeros(2, L.page_bytes_quantized(d), dtype=torch.uint8, device="cuda")
    L.quantize_latents(d, cache[n - 2:].contiguous().view(torch.uint8), i32([[1, 0]]), i32([0]), i32([128]), 128, small, i32([[0, 1]]))
    assert torch.equal(out[n - 3], small[0]) and torch.equal(out[n - 1], small[1]) and int(out[:n - 3].max()) == 0
