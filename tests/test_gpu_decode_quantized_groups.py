"""Decode attention over 8-bit pages whose value groups differ in size, and scores of any size."""
import numpy as np
import pytest

import lorc_inputs as gen
from test_gpu_decode_quantized import SHAPES, Cache8
from test_gpu_decode_quantized_sequences import check_each

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["absorbed 8b", "absorbed wide values", "absorbed rank 1024", "rotary 8b", "rotary groups of 8", "rotary wide values", "rotary rank 1024",
                                  "rotary groups of 12", "rotary d 64"])
def test_groups_of_values_of_different_sizes(name):
    """Value latents of every other group are 2^-16 of the rest and the value factor's rows as much larger, so that all groups weigh the
    same in the output.  In the 2^-16 group a weight 2^-j of the largest is 2^(-16 - j) of the largest product of weight and scale: it has to
    keep its bits.  (2^8 and 2^-8: the partial rows are fp16.)"""
    import torch
    shape = SHAPES[name]
    r_v = shape.get("r_v", 512)
    size = np.where(np.arange(r_v) // 128 % 2 == 1, 2.0 ** -8, 2.0 ** 8)[None]
    c = Cache8(ctx=[500, 1, 77, 1300], seed=33, amp_v=lambda rng, n: size, **shape)
    c.B_v = (c.B_v / size.T).astype(np.float32)          # powers of two: still bf16 values
    bf = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(torch.bfloat16).contiguous()  # noqa: E731
    c.packed = c.L.pack_factors(c.desc, bf(np.zeros((64, c.desc.rank_k))), bf(np.zeros((64, r_v))), bf(c.B_k), bf(c.B_v))
    assert np.array_equal(gen.bf16_round(c.B_v), c.B_v)
    check_each(c)


@pytest.mark.parametrize("name", ["plain 8b", "plain groups of 20"])
def test_heads_of_values_of_different_sizes(name):
    """An uncompressed layer's groups are its KV heads: each by itself."""
    n_kv = SHAPES[name].get("h_kv", 8)
    size = np.repeat(np.where(np.arange(n_kv) % 2 == 1, 2.0 ** -8, 2.0 ** 8), 128)[None]
    check_each(Cache8(ctx=[500, 1, 77, 1300], seed=34, amp_v=lambda rng, n: size, **SHAPES[name]), heads=True)


@pytest.mark.parametrize("name", ["plain 8b", "absorbed 8b", "absorbed rank 1024", "rotary 8b", "rotary rank 1024"])
def test_scores_of_any_size_stay_finite(name):
    """Scores of up to 2^27: a softmax of one position or two, whose reference fp32 rounds by several units of the exponent.  (Scaled queries
    and keys stay below the largest fp16.)"""
    import torch
    for power in range(0, 12):
        c = Cache8(ctx=[300, 65], seed=35, scale=2.0 ** 12, amp_k=2.0 ** power, **SHAPES[name])
        assert bool(torch.isfinite(c.call()).all()), power
