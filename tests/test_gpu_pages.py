"""The page calls against the oracle, entry for entry: random turns of a pool's life, lists longer than a plan's threads, pools longer
than one pass of a plan, refused and short entries, and copies of pages of any size."""
import numpy as np
import pytest

from oracle import cache_oracle as co

pytestmark = pytest.mark.gpu


def dev32(v):
    import torch
    return torch.as_tensor(np.ascontiguousarray(v, np.int32)).cuda()


class Pool:
    """The same state on the device and in the oracle; every call compares all of it."""

    def __init__(self, n_seqs, max_pages, n_pages, table=None, refs=None, misaligned=False):
        import torch
        import paper_2410_03111_amd as L
        self.L, self.torch = L, torch
        self.o = co.Pages(np.full((n_seqs, max_pages), -1) if table is None else table, np.zeros(n_pages) if refs is None else refs)
        self.table = dev32(self.o.table)
        room = torch.zeros(n_pages + 1, dtype=torch.int32, device="cuda")
        self.refs = room[1:] if misaligned else room[:n_pages]
        self.refs.copy_(dev32(self.o.refs))

    def same(self, what=""):
        assert np.array_equal(self.table.cpu().numpy(), self.o.table), what
        assert np.array_equal(self.refs.cpu().numpy(), self.o.refs), what

    def fork(self, parents, children, lens):
        n = len(parents)
        src, dst, status = (dev32(np.full(n, 77)) for _ in range(3))
        self.L.fork_sequences(self.table, self.refs, dev32(parents), dev32(children), dev32(lens), src, dst, status)
        want = self.o.fork(list(map(int, parents)), list(map(int, children)), list(map(int, lens)))
        for got, ref, name in zip((src, dst, status), want, ("src", "dst", "status")):
            assert got.cpu().tolist() == ref, name
        self.same("fork")
        return want

    def free(self, seqs):
        self.L.free_sequences(self.table, self.refs, dev32(seqs))
        self.o.free(seqs)
        self.same("free")

    def compact(self, max_moves):
        src, dst = (dev32(np.full(max_moves, 77)) for _ in range(2))
        new = dev32(np.full(len(self.o.refs), 77))
        self.L.compact_pages(self.table, self.refs, src, dst, new)
        want = self.o.compact(max_moves)
        assert src.cpu().tolist() == want[0] and dst.cpu().tolist() == want[1]
        assert np.array_equal(new.cpu().numpy(), want[2])
        self.same("compact")
        return want

    def reserve(self, seqs, lens):
        status = dev32(np.full(len(seqs), 77))
        self.L.reserve_pages(self.table, self.refs, dev32(seqs), dev32(lens), status)
        want = self.o.reserve(list(map(int, seqs)), list(map(int, lens)))
        assert status.cpu().tolist() == want
        self.same("reserve")
        return want


@pytest.mark.parametrize("seed, n_seqs, max_pages, n_pages", [(0, 12, 6, 25), (1, 3, 1, 2), (2, 70, 67, 900), (3, 9, 130, 40)])
def test_random_turns(seed, n_seqs, max_pages, n_pages):
    rng = np.random.default_rng(seed)
    pool = Pool(n_seqs, max_pages, n_pages, misaligned=seed % 2 == 1)
    row = lambda n: rng.integers(-1, n_seqs + 1, n)  # noqa: E731
    length = lambda n: np.where(rng.random(n) < 0.3, 64 * rng.integers(0, max_pages + 1, n), rng.integers(-2, 64 * max_pages + 3, n))  # noqa: E731
    for _ in range(60):
        n = int(rng.integers(1, 9))
        kind = rng.integers(5)
        if kind == 0:
            pool.reserve(row(n), length(n))
        elif kind <= 2:
            pool.fork(row(n), row(n), length(n))
        elif kind == 3:
            pool.free([int(s) for s in row(n)])
        else:
            pool.compact(int(rng.integers(0, n_pages)))
    pool.compact(n_pages)


def test_lists_longer_than_a_plan_and_pools_longer_than_a_pass():
    n_seqs, max_pages, n_pages = 2600, 20, 70001       # a plan has 1024 threads and walks 16384 pages at a time
    rng = np.random.default_rng(5)
    pool = Pool(n_seqs, max_pages, n_pages)
    assert set(pool.reserve(np.arange(1300), rng.integers(1, 64 * max_pages, 1300))) == {co.OK}
    pool.free([int(s) for s in rng.permutation(1300)[:200]])
    order = rng.permutation(np.arange(1300, 2600))
    want = pool.fork(rng.integers(0, 1300, 1300), order, rng.integers(0, 64 * max_pages, 1300))
    assert set(want[2]) == {co.OK}
    pool.free(list(range(0, 1300, 2)))
    pool.compact(100)
    pool.compact(n_pages // 2)
    pool.reserve(np.arange(0, 1300, 2), np.full(650, 64 * max_pages))


def test_scattered_pages_over_several_passes():
    rng = np.random.default_rng(6)
    n_seqs, max_pages, n_pages = 50, 400, 50000
    ids = rng.permutation(n_pages)[:n_seqs * max_pages].reshape(n_seqs, max_pages)
    refs = np.zeros(n_pages, np.int32)
    refs[ids] = 1
    pool = Pool(n_seqs, max_pages, n_pages, ids, refs)
    pool.fork([3] * 10 + [7], list(range(10, 20)) + [3], [100] * 11)     # rows in use: refused
    pool.free(list(range(10, 20)))
    want = pool.fork([3] * 10, range(10, 20), [64 * 400 - 1] * 10)
    assert want[2] == [co.OK] * 10
    moved = pool.compact(n_pages // 2)
    assert sum(v >= 0 for v in moved[0]) > 1000
    used = np.flatnonzero(pool.o.refs > 0)
    assert np.array_equal(used, np.arange(len(used)))


def test_pages_run_out_in_order():
    pool = Pool(6, 4, 5)
    assert pool.reserve([0, 1, 2, 3], [65, 129, 1, 0]) == [co.OK, co.OK, co.SHORT, co.OK]      # 2 + 3 pages, none left, none needed
    assert pool.fork([0, 1, 0], [4, 5, 2], [64, 70, 65])[2] == [co.OK, co.SHORT, co.SHORT]
    pool.free([1, 1])                                                                          # once
    assert pool.fork([0, 0, 1], [1, 2, 3], [65, 1, 1])[2] == [co.OK, co.OK, co.REFUSED]        # 1 is a child here
    assert pool.reserve([5, 5, -1, 6, 0], [64, 64, 1, 1, 1000]) == [co.OK, co.REFUSED, co.REFUSED, co.REFUSED, co.REFUSED]


def test_a_fork_of_unmapped_entries_and_ids_outside_the_pool():
    pool = Pool(4, 4, 10, [[3, 99, -7, 5], [-1] * 4, [-5, 1, -1, -1], [12, -1, -1, -1]], [0, 1, 0, 1, 0, 1, 0, 0, 0, 0])
    assert pool.fork([0, 0, 0], [1, 2, 3], [256, 65, 130])[2] == [co.OK] * 3      # unmapped tails: nothing to copy
    pool.free([0])
    pool.compact(5)


@pytest.mark.parametrize("page_bytes, n_pages", [(16, 9), (48, 33), (16384, 5), (16400, 7), (66048, 40), (131072, 21), (33024, 3)])
def test_copies(page_bytes, n_pages):
    import torch
    import paper_2410_03111_amd as L
    rng = np.random.default_rng(page_bytes)
    data = rng.integers(0, 256, (n_pages, page_bytes), dtype=np.uint8)
    order = rng.permutation(n_pages)
    n = n_pages // 2
    src, dst = order[:n].copy(), order[n:2 * n].copy()
    src = np.concatenate([src, [-1, 0, n_pages, order[-1], 2]])
    dst = np.concatenate([dst, [0, -1, 0, order[-1], n_pages]])        # skipped
    pool = torch.from_numpy(data.copy()).cuda()
    L.copy_pages(pool, dev32(src), dev32(dst))
    want = data.copy()
    want[dst[:n]] = data[src[:n]]
    assert np.array_equal(pool.cpu().numpy(), want)
    flat = torch.from_numpy(data.copy()).cuda().view(-1)
    L.copy_pages(flat, dev32(src), dev32(dst), page_bytes=page_bytes)
    assert np.array_equal(flat.cpu().numpy().reshape(n_pages, page_bytes), want)


def test_copies_beyond_4_gib():
    import torch
    import paper_2410_03111_amd as L
    pool = torch.zeros(70, 1 << 24, dtype=torch.int32, device="cuda")       # 64 MiB pages
    pool[68] = 5
    pool[2] = 9
    L.copy_pages(pool, dev32([68, 2]), dev32([1, 69]))
    assert bool((pool[1] == 5).all()) and bool((pool[69] == 9).all()) and int(pool[0].sum()) == 0 and int(pool[67].sum()) == 0


def test_calls_replay_from_a_graph_on_another_stream():
    import torch
    import paper_2410_03111_amd as L
    table0 = np.full((6, 4), -1, np.int32)
    table0[0, :3] = [7, 2, 5]
    refs0 = np.zeros(12, np.int32)
    refs0[[7, 2, 5]] = 1
    parents, children, lens = dev32([0, 0]), dev32([1, 2]), dev32([150, 128])
    table, refs, t0, r0 = dev32(table0), dev32(refs0), dev32(table0), dev32(refs0)
    src, dst, status, new, gone = dev32([0, 0]), dev32([0, 0]), dev32([0, 0]), dev32(np.zeros(12)), dev32([0])
    msrc, mdst = dev32(np.zeros(6)), dev32(np.zeros(6))
    pool0 = torch.arange(12 * 1024, dtype=torch.int32, device="cuda").view(12, 1024)
    pool = pool0.clone()
    ws = torch.empty(L.pages_workspace_bytes(6, 12), dtype=torch.uint8, device="cuda")

    def turn():
        table.copy_(t0), refs.copy_(r0), pool.copy_(pool0)
        L.fork_sequences(table, refs, parents, children, lens, src, dst, status, workspace=ws)
        L.copy_pages(pool, src, dst)
        L.free_sequences(table, refs, gone)
        L.compact_pages(table, refs, msrc, mdst, new)
        L.copy_pages(pool, msrc, mdst)
        L.reserve_pages(table, refs, gone, lens[:1], status[:1], workspace=ws)

    turn()
    torch.cuda.synchronize()
    results = lambda: [t.cpu().numpy().copy() for t in (table, refs, src, dst, status, new, msrc, mdst, pool)]  # noqa: E731
    eager = results()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            turn()
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        for t in (table, refs, src, dst, status, new, msrc, mdst, pool):
            t.fill_(rep)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(results(), eager):
            assert np.array_equal(a, b), rep


def test_refused_arguments():
    import torch
    import paper_2410_03111_amd as L
    table, refs, row, other = dev32(np.full((4, 3), -1)), dev32(np.zeros(9)), dev32([0, 1]), dev32([2, 3])
    src, dst, status = dev32([0, 0]), dev32([0, 0]), dev32([0, 0])
    ws = torch.empty(L.pages_workspace_bytes(4, 9), dtype=torch.uint8, device="cuda")
    good = {L.fork_sequences: dict(block_table=table, page_refs=refs, parents=row, children=other, lens=row, copy_src=src, copy_dst=dst, status=status, workspace=ws),
            L.free_sequences: dict(block_table=table, page_refs=refs, seqs=row),
            L.compact_pages: dict(block_table=table, page_refs=refs, move_src=src, move_dst=dst, page_map=dev32(np.zeros(9))),
            L.reserve_pages: dict(block_table=table, page_refs=refs, seqs=row, lens=row, status=status, workspace=ws)}
    for call, args in good.items():
        call(**args)
        for key, t in args.items():
            wide = torch.zeros(t.shape[0] * 2, *t.shape[1:], dtype=t.dtype, device="cuda")
            for bad in (t.cpu(), t.to(torch.int64), wide[::2], None if key != "workspace" else 5):
                with pytest.raises(TypeError):
                    call(**{**args, key: bad})
            if key not in ("block_table", "page_refs", "seqs", "parents", "workspace", "move_src"):
                with pytest.raises(ValueError):
                    call(**{**args, key: wide})
        if "workspace" in args:
            with pytest.raises(L.LorcError):
                call(**{**args, "workspace": ws[:-1]})
    pool = torch.zeros(9, 32, dtype=torch.uint8, device="cuda")
    L.copy_pages(pool, row, other)
    for bad, error in ((dict(pool=pool.cpu()), TypeError), (dict(pool=pool[:, ::2]), TypeError), (dict(src=row.to(torch.int64)), TypeError), (dict(dst=other[:1]), ValueError),
                       (dict(pool=pool[:0]), ValueError), (dict(page_bytes=24), L.LorcError), (dict(page_bytes=0), L.LorcError), (dict(page_bytes=-16), L.LorcError),
                       (dict(page_bytes=512), L.LorcError), (dict(pool=pool.view(-1)[8:-24].view(8, 32)), L.LorcError)):
        with pytest.raises(error):
            L.copy_pages(**{**dict(pool=pool, src=row, dst=other), **bad})


def test_two_graphs_share_a_workspace():
    import torch
    import paper_2410_03111_amd as L
    ws = torch.empty(L.pages_workspace_bytes(5000, 700), dtype=torch.uint8, device="cuda")      # a table beyond what a small plan holds
    rng, graphs, pools = np.random.default_rng(3), [], []
    for g in range(2):
        pool = Pool(5000, 4, 700)
        rows = rng.permutation(5000)[:120]
        pool.reserve(rows, rng.integers(0, 257, 120))
        args = rows[:40], np.setdiff1d(np.arange(5000), rows)[:40], rng.integers(0, 257, 40)
        lists = [dev32(a) for a in args] + [dev32(np.full(40, 77)) for _ in range(3)]
        keep = pool.table.clone(), pool.refs.clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            pool.table.copy_(keep[0]), pool.refs.copy_(keep[1])
            L.fork_sequences(pool.table, pool.refs, *lists, workspace=ws)
        want = pool.o.fork(*[list(map(int, a)) for a in args])
        graphs.append(graph)
        pools.append((pool, lists, want, keep))
    for rep in range(3):
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for pool, lists, want, _ in pools:
            pool.same(rep)
            assert [t.cpu().tolist() for t in lists[3:]] == [list(w) for w in want]
        ws.fill_(255)
