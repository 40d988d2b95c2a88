"""CPU tests of the page calls and of the 8-bit cache's entry points: sizes and index helpers against the oracle's formulas, and every
refusal that the host decides (nothing here reaches a device)."""
import ctypes
import os
import re

import pytest

from oracle import cache_oracle as co

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
L = pytest.importorskip("paper_2410_03111_amd", reason="liblorc.so not built: python paper_2410_03111_amd/build.py")
lib = L._lib
P = ctypes.c_void_p(4096)       # a pointer of good alignment that no refused call follows
ODD = ctypes.c_void_p(4100)


def desc(**kw):
    d = dict(d_model=4096, n_q_heads=32, n_kv_heads=8, head_dim=128, rank_k=512, rank_v=512, rope_base=1e4)
    d.update(kw)
    return L.layer_desc(**d)


@pytest.mark.parametrize("r_k, r_v", [(32, 32), (128, 160), (512, 512), (1024, 96)])
def test_page_size_and_scale_bytes(r_k, r_v):
    d = desc(rank_k=r_k, rank_v=r_v)
    assert L.page_bytes_quantized(d) == co.page_size(r_k, r_v)
    seen = set()
    for slot in (0, 1, 31, 32, 63):
        for r, value, at in ((r_k, False, L.cache_scale_index_k), (r_v, True, L.cache_scale_index_v)):
            for j in (0, 1, 127, 128, r - 1):
                if j < r:
                    assert at(d, slot, j) == co.scale_index(r_k, r_v, slot, j, value)
                    assert 64 * (r_k + r_v) <= at(d, slot, j) < L.page_bytes_quantized(d)
                    seen.add((value, slot, j // 128, at(d, slot, j)))
            assert at(d, slot, r) == -1 and at(d, slot, -1) == -1
    assert len({s[-1] for s in seen}) == len({s[:3] for s in seen}) and L.cache_scale_index_k(d, 64, 0) == -1
    assert L.page_bytes_quantized(desc(rank_k=48)) == 0 and L.cache_scale_index_v(desc(rank_k=48), 0, 0) == -1


def test_status_values_of_the_header():
    header = open(os.path.join(ROOT, "include", "lorc.h")).read()
    found = dict(re.findall(r"#define (LORC_PAGES_[A-Z]+) (\d)", header))
    assert found == {"LORC_PAGES_OK": str(L.PAGES_OK), "LORC_PAGES_REFUSED": str(L.PAGES_REFUSED), "LORC_PAGES_SHORT": str(L.PAGES_SHORT)}
    assert (co.OK, co.REFUSED, co.SHORT) == (L.PAGES_OK, L.PAGES_REFUSED, L.PAGES_SHORT)


def test_copy_pages_refusals():
    ok = dict(pool=P, page_bytes=4096, n_pages=8, src=P, dst=P, count=1)
    for bad in (dict(pool=None), dict(pool=ODD), dict(page_bytes=0), dict(page_bytes=4100), dict(n_pages=0), dict(src=None), dict(dst=None), dict(count=-1),
                dict(page_bytes=1 << 40, count=1 << 20)):
        assert lib.lorc_copy_pages(*{**ok, **bad}.values(), None) == L.EINVAL, bad
    assert lib.lorc_copy_pages(*{**ok, "count": 0}.values(), None) == L.OK


def test_table_call_refusals():
    need = L.pages_workspace_bytes(4, 100)
    assert need > 0 and L.pages_workspace_bytes(0, 100) == 0 and L.pages_workspace_bytes(4, 0) == 0
    table = dict(block_table=P, n_seqs=4, max_pages=8, page_refs=P, n_pages=100)
    calls = {
        "lorc_fork_sequences": dict(table, parents=P, children=P, lens=P, n=2, copy_src=P, copy_dst=P, status=P, workspace=P, workspace_bytes=need),
        "lorc_free_sequences": dict(table, seqs=P, n=2),
        "lorc_compact_pages": dict(table, move_src=P, move_dst=P, max_moves=3, page_map=P),
        "lorc_reserve_pages": dict(table, seqs=P, lens=P, n=2, status=P, workspace=P, workspace_bytes=need),
    }
    for name, args in calls.items():
        fn = getattr(lib, name)
        for key, value in args.items():
            if value is P:
                assert fn(*{**args, key: None}.values(), None) == L.EINVAL, (name, key)
        for bad in (dict(n_seqs=0), dict(max_pages=0), dict(n_pages=-1), dict(max_pages=(1 << 31) - 1)):
            assert fn(*{**args, **bad}.values(), None) == L.EINVAL, (name, bad)
        count = "max_moves" if "max_moves" in args else "n"
        assert fn(*{**args, count: -1}.values(), None) == L.EINVAL, name
        if "workspace" in args:
            assert fn(*{**args, "workspace": ODD}.values(), None) == L.EINVAL, name
            assert fn(*{**args, "workspace_bytes": need - 1}.values(), None) == L.EWORKSPACE, name
        if "n" in args:
            assert fn(*{**args, "n": 0}.values(), None) == L.OK, name


def test_quantize_refusals():
    d = desc()
    args = dict(desc=ctypes.byref(d), cache=P, block_table=P, max_pages=4, n_pages=9, pos_begin=P, pos_end=P, b=2, max_tokens=5, cache_q8=P,
                block_table_q8=P, max_pages_q8=4, n_pages_q8=9)
    call = lambda **kw: lib.lorc_quantize_latents(*{**args, **kw}.values(), None)  # noqa: E731
    for key, value in args.items():
        if value is P:
            assert call(**{key: None}) == L.EINVAL, key
    for bad in (dict(desc=None), dict(b=0), dict(max_tokens=-1), dict(max_pages=0), dict(n_pages=0), dict(max_pages_q8=0), dict(n_pages_q8=0), dict(cache=ODD),
                dict(cache_q8=ODD), dict(b=1 << 30, max_tokens=1 << 30, max_pages=1 << 20, max_pages_q8=1 << 20)):
        assert call(**bad) == L.EINVAL, bad
    assert call(desc=ctypes.byref(desc(rank_k=40))) == L.EUNSUPPORTED
    assert call(max_tokens=0) == L.OK


FORMS = {
    "lorc_decode_attention_quantized": (True, L.decode_quantized_workspace_bytes, desc()),
    "lorc_decode_attention_plain_quantized": (True, L.decode_plain_quantized_workspace_bytes, desc(rank_k=1024, rank_v=1024)),
    "lorc_decode_attention_absorbed_quantized": (False, L.decode_absorbed_quantized_workspace_bytes, desc()),
}


@pytest.mark.parametrize("name", FORMS)
def test_decode_refusals(name):
    rotary, size, d = FORMS[name]
    args = dict(desc=ctypes.byref(d), q=P, **(dict(q_pos=P) if rotary else {}), ctx_len=P, b=2, max_ctx=100, packed=P, cache=P, block_table=P, max_pages=2, n_pages=9,
                out=P, workspace=P, workspace_bytes=size(d, 2, 100))
    call = lambda **kw: getattr(lib, name)(*{**args, **kw}.values(), None)  # noqa: E731
    for key, value in args.items():
        if value is P:
            assert call(**{key: None}) == L.EINVAL, key
    for bad in (dict(desc=None), dict(b=0), dict(max_ctx=-1), dict(max_pages=0), dict(max_pages=1), dict(n_pages=0), dict(q=ODD), dict(cache=ODD), dict(out=ODD),
                dict(workspace=ODD), dict(packed=ODD)):
        assert call(**bad) == L.EINVAL, bad
    unsupported = [desc(rank_k=2048, n_q_heads=64, n_kv_heads=32, d_model=8192), desc(rank_v=2048, n_q_heads=64, n_kv_heads=32, d_model=8192), desc(head_dim=96)]
    if "plain" in name:
        unsupported += [desc(rank_k=512, rank_v=1024), desc(head_dim=64, rank_k=512, rank_v=512)]
    for u in unsupported:
        assert size(u, 2, 100) == 0 and call(desc=ctypes.byref(u)) == L.EUNSUPPORTED


@pytest.mark.parametrize("name", FORMS)
def test_a_workspace_for_a_larger_call_holds_one_split_of_every_smaller_one(name):
    _, size, d = FORMS[name]
    width = 128 if "plain" in name else 512
    for b, ctx in ((1, 0), (1, 64), (3, 1000), (16, 4096), (64, 777), (64, 100000)):
        least = b * 32 * 8 + b * 32 * width * 2
        assert all(size(d, b2, ctx2) >= least for b2 in (b, b + 1, 2 * b) for ctx2 in (ctx, ctx + 65, 2 * ctx + 4096))
        assert size(d, b, -1) == 0 and size(d, 0, ctx) == 0


@pytest.mark.parametrize("name", FORMS)
def test_contexts_beyond_what_512_splits_walk_are_refused(name):
    rotary, size, d = FORMS[name]
    most = {True: 512 * 128 * 64, False: 1 << 30}["_attention_quantized" in name]   # a rotary split walks up to 128 pages
    if "absorbed" in name:
        most = 512 * 1024 * 64
    args = dict(desc=ctypes.byref(d), q=P, **(dict(q_pos=P) if rotary else {}), ctx_len=P, b=1, max_ctx=0, packed=P, cache=P, block_table=P, max_pages=1 << 25, n_pages=9,
                out=P, workspace=P, workspace_bytes=1 << 40)
    assert size(d, 1, most) > 0
    for ctx in (most + 1, 2 ** 31 - 64, 2 ** 31 - 1):
        assert size(d, 1, ctx) == 0
        assert getattr(lib, name)(*{**args, "max_ctx": ctx}.values(), None) == L.EUNSUPPORTED


def test_tables_counts_and_lists_beyond_2_to_the_30_are_refused():
    table = dict(block_table=P, n_seqs=4, max_pages=8, page_refs=P, n_pages=100)
    for name, args, count in (("lorc_fork_sequences", dict(parents=P, children=P, lens=P, n=0, copy_src=P, copy_dst=P, status=P, workspace=P, workspace_bytes=1 << 40), "n"),
                              ("lorc_free_sequences", dict(seqs=P, n=0), "n"),
                              ("lorc_compact_pages", dict(move_src=P, move_dst=P, max_moves=0, page_map=P), "max_moves"),
                              ("lorc_reserve_pages", dict(seqs=P, lens=P, n=0, status=P, workspace=P, workspace_bytes=1 << 40), "n")):
        for bad in (dict(n_pages=(1 << 30) + 1), dict(n_seqs=(1 << 30) // 8 + 1), dict(n_seqs=2 ** 31 - 1), {count: (1 << 30) + 1}):
            assert getattr(lib, name)(*{**table, **args, **bad}.values(), None) == L.EINVAL, (name, bad)


@pytest.mark.parametrize("which", ["max_pages", "max_pages_q8"])
def test_positions_of_a_quantized_table_stay_below_2_to_the_31(which):
    d = desc()
    args = dict(desc=ctypes.byref(d), cache=P, block_table=P, max_pages=4, n_pages=9, pos_begin=P, pos_end=P, b=2, max_tokens=0, cache_q8=P,
                block_table_q8=P, max_pages_q8=4, n_pages_q8=9)
    assert lib.lorc_quantize_latents(*args.values(), None) == L.OK
    assert lib.lorc_quantize_latents(*{**args, which: 1 << 25}.values(), None) == L.EINVAL
