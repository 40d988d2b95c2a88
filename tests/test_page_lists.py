"""CPU tests of the page calls' lists: empty ones, whose tensors have no address, and counts beyond the limit."""
import ctypes

import pytest

L = pytest.importorskip("paper_2410_03111_amd", reason="liblorc.so not built: python paper_2410_03111_amd/build.py")
lib = L._lib
P = ctypes.c_void_p(4096)       # a pointer of good alignment that no refused call follows
TABLE = dict(block_table=P, n_seqs=4, max_pages=8, page_refs=P, n_pages=100)
CALLS = {
    "lorc_copy_pages": (dict(pool=P, page_bytes=4096, n_pages=8), dict(src=None, dst=None, count=0), "count"),
    "lorc_fork_sequences": (TABLE, dict(parents=None, children=None, lens=None, n=0, copy_src=None, copy_dst=None, status=None, workspace=P, workspace_bytes=1 << 40), "n"),
    "lorc_free_sequences": (TABLE, dict(seqs=None, n=0), "n"),
    "lorc_reserve_pages": (TABLE, dict(seqs=None, lens=None, n=0, status=None, workspace=P, workspace_bytes=1 << 40), "n"),
}


@pytest.mark.parametrize("name", CALLS)
def test_a_list_of_no_entries_needs_no_pointer(name):
    state, lists, count = CALLS[name]
    call = lambda **kw: getattr(lib, name)(*{**state, **lists, **kw}.values(), None)  # noqa: E731
    assert call() == L.OK
    for key, value in state.items():        # what is not a list is checked all the same
        if value is P:
            assert call(**{key: None}) == L.EINVAL, key
    assert call(**{count: 1}) == L.EINVAL


@pytest.mark.parametrize("name", CALLS)
def test_counts_beyond_the_limit(name):
    state, lists, count = CALLS[name]
    given = {k: P if v is None else v for k, v in lists.items()}
    for bad in ((1 << 30) + 1, 2 ** 31 - 1, -1):
        assert getattr(lib, name)(*{**state, **given, count: bad}.values(), None) == L.EINVAL
