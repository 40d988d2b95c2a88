"""Calls that need more work-items than a launch holds (2^32): lists of that many entries, and prompts of that many pages.  The entries that
do something lie at both ends."""
import numpy as np
import pytest

from oracle import cache_oracle as co
from test_gpu_pages import Pool, dev32

pytestmark = pytest.mark.gpu


def at_the_ends(n, values):
    """n entries of -1, with `values` over both ends."""
    import torch
    t = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    half = len(values) // 2
    t[:half] = dev32(values[:half])
    t[n - (len(values) - half):] = dev32(values[half:])
    return t


def test_copies_of_more_pieces_than_a_launch_holds():
    import torch
    import paper_2410_03111_amd as L
    pool = torch.arange(64, dtype=torch.int32, device="cuda")[:, None].repeat(1, 4).contiguous()       # pages of 16 bytes
    want = pool.clone()
    want[[9, 10, 11, 12]] = want[[1, 2, 3, 4]]
    n = (1 << 24) + 5
    L.copy_pages(pool, at_the_ends(n, [1, 2, 3, 4]), at_the_ends(n, [9, 10, 11, 12]))
    assert torch.equal(pool, want)


def test_forks_and_releases_of_more_rows_than_a_launch_holds():
    import torch
    import paper_2410_03111_amd as L
    n = (1 << 26) + 7
    pool = Pool(8, 3, 40)
    pool.reserve([0, 1], [150, 64])
    args = [0, 1, 0, 1], [2, 3, 4, 5], [130, 64, 150, 20]
    lists = [at_the_ends(n, v) for v in args]
    out = [torch.full((n,), 77, dtype=torch.int32, device="cuda") for _ in range(3)]
    L.fork_sequences(pool.table, pool.refs, *lists, *out)
    want = pool.o.fork(*args)
    pool.same()
    for got, ref, fill in zip(out, want, (-1, -1, co.REFUSED)):
        assert got[:2].tolist() + got[-2:].tolist() == ref
        assert bool((got[2:-2] == fill).all())
    L.free_sequences(pool.table, pool.refs, at_the_ends(n, [0, 2, 5, 0]))
    pool.o.free([0, 2, 5])
    pool.same()


def test_reservations_of_more_rows_than_a_launch_holds():
    import torch
    import paper_2410_03111_amd as L
    n = (1 << 28) + 3
    pool = Pool(8, 3, 40)
    args = [3, 0, 3, 5], [70, 192, 10, 1]
    lists = [at_the_ends(n, v) for v in args]
    status = torch.full((n,), 77, dtype=torch.int32, device="cuda")
    L.reserve_pages(pool.table, pool.refs, *lists, status)
    want = pool.o.reserve(*args)
    pool.same()
    assert status[:2].tolist() + status[-2:].tolist() == want and bool((status[2:-2] == co.REFUSED).all())


def test_quantizing_more_pages_than_a_launch_holds():
    import torch
    import paper_2410_03111_amd as L
    desc = L.layer_desc(64, 4, 2, 64, 32, 32, 1e4)
    b, max_pages = 8200, 1100                # two workgroups per page: 18.0 million of 256 threads
    page, page_q8 = L.page_bytes(desc), L.page_bytes_quantized(desc)
    cache = torch.randn(4 * page // 2, device="cuda").to(torch.bfloat16).view(torch.uint8)
    table = torch.full((b, max_pages), -1, dtype=torch.int32, device="cuda")
    table[0, 0], table[-1, 0], table[-1, -1] = 2, 0, 3
    begin, end = (torch.zeros(b, dtype=torch.int32, device="cuda") for _ in range(2))
    end[0], end[-1] = 50, 64 * max_pages
    out = [torch.full((4 * page_q8,), 0x55, dtype=torch.uint8, device="cuda") for _ in range(2)]
    L.quantize_latents(desc, cache, table, begin, end, 64 * max_pages, out[0], table)
    for s in (0, b - 1):
        L.quantize_latents(desc, cache, table[s:s + 1], begin[s:s + 1], end[s:s + 1], 64 * max_pages, out[1], table[s:s + 1])
    assert torch.equal(out[0], out[1]) and bool((out[0].view(4, -1)[1] == 0x55).all()) and bool((out[0].view(4, -1)[3] != 0x55).any())


def test_a_batch_of_more_workgroups_than_a_launch_holds_is_refused():
    import torch
    import paper_2410_03111_amd as L
    desc, b = L.layer_desc(64, 1, 1, 128, 128, 128, 1e4), 1 << 24
    new = lambda n, dtype: torch.zeros(n, dtype=dtype, device="cuda")  # noqa: E731
    q, out = torch.zeros(b, 1, 128, dtype=torch.bfloat16, device="cuda"), torch.full((b, 1, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    rows = torch.full((b, 1), -1, dtype=torch.int32, device="cuda")
    packed, pool = new(L.packed_bytes(desc), torch.uint8), new(2 * L.page_bytes_quantized(desc), torch.uint8)
    ws = new(L.decode_plain_quantized_workspace_bytes(desc, b, 64), torch.uint8)
    with pytest.raises(L.LorcError) as e:
        L.decode_attention_plain_quantized(desc, q, rows.view(-1), rows.view(-1), 64, packed, pool, rows, out=out, workspace=ws)
    assert e.value.code == L.EINVAL and bool((out == 7.0).all())
