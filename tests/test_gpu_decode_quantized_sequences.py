"""Decode attention over 8-bit pages, every sequence by itself: a batch's norm is that of its shortest sequences, whose outputs are the
largest (nothing is averaged), and would hide what goes wrong in long ones.  Tolerances: those of test_gpu_decode_quantized.py, which are
derived for every output row."""
import numpy as np
import pytest

from lorc_testlib import TOL
from test_gpu_decode_quantized import LENGTHS, NORM2, SHAPES, Cache8

pytestmark = pytest.mark.gpu


def check_each(c, got=None, heads=False):
    """heads: every query head by itself."""
    got, ref = (c.call() if got is None else got).float().cpu().numpy().astype(np.float64), c.oracle()
    assert np.all(np.isfinite(got))
    for s, n in enumerate(c.ctx):
        for h in range(c.h_q) if heads else [slice(None)]:
            a, b = got[s, h], ref[s, h]
            if n == 0:
                assert np.all(a == 0.0)
                continue
            n2, mx = np.linalg.norm(a - b) / np.linalg.norm(b), np.abs(a - b).max() / np.abs(b).max()
            assert n2 <= NORM2 and mx <= TOL, (s, n, h, n2, mx)


@pytest.mark.parametrize("ctx", [LENGTHS, [1700], [1, 2500, 700, 1337]], ids=["lengths", "one", "ragged"])
@pytest.mark.parametrize("name", SHAPES)
def test_every_sequence(name, ctx):
    check_each(Cache8(ctx=ctx, seed=31, **SHAPES[name]))


# pages that a split walks at most, and a layer for each kernel with such a limit
FULL = {"rotary": (128, dict(form="rotary", h_q=8, h_kv=2, r_k=96, r_v=64)),
        "rotary, groups of 12": (128, dict(form="rotary", h_q=24, h_kv=2, r_k=64, r_v=32)),
        "rotary, rank 608": (128, dict(form="rotary", h_q=10, h_kv=5, r_k=608, r_v=32)),
        "rotary, d 64": (128, dict(form="rotary", h_q=6, h_kv=3, d=64, r_k=64, r_v=96)),
        "absorbed": (1024, dict(form="absorbed", h_q=4, h_kv=2, d=64, r_k=32, r_v=32))}


@pytest.mark.parametrize("name", FULL)
def test_splits_of_the_most_pages(name):
    """The workspace holds the fewest splits that the kernel can do with: two, of as many pages as a split can have (the last ones less)."""
    import torch
    pages, shape = FULL[name]
    c = Cache8(ctx=[2 * 64 * pages - 21, 64 * pages + 1], seed=32, **shape)
    size = sum(-(-2 * 2 * c.h_q * width // 256) * 256 for width in (8, 2 * c.desc.rank_v))
    check_each(c, got=c.call(workspace=torch.empty(size, dtype=torch.uint8, device="cuda")))
    with pytest.raises(c.L.LorcError) as e:
        c.call(workspace=torch.empty(size - 256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == c.L.EWORKSPACE
