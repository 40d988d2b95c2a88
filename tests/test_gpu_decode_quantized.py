"""Decode attention over 8-bit pages against fp64 on the values that the pages stand for.

Tolerances.  The outputs are bf16: rounding to nearest is off by at most half a step, 2^-8 of the value, and by 2^-8 / sqrt(3) = 2.3e-3
in the 2-norm where errors are spread evenly over the worst binade.  Queries, rotated keys, weights and split partials are fp16 (half
a step 2^-11, 2.8e-4 in the 2-norm each); rounded queries and keys move a score in log2 units by about 2 x 2.8e-4 x ||q o k||, of size
1.44 for N(0, 1) keys and queries, and a weight by ln 2 of that, 5.6e-4, its normaliser once more.  In quadrature
sqrt(2.3^2 + 4 x 0.28^2 + 2 x 0.56^2) = 2.5e-3; twice that is allowed in the 2-norm, and 2e-2 of the largest output at any place (the
bound of the bf16 paths)."""
import numpy as np
import pytest

import lorc_inputs as gen
from lorc_testlib import PAGE, TOL, page_gather_indices
from oracle import cache_oracle as co
from oracle import lorc_oracle as orc

pytestmark = pytest.mark.gpu
NORM2 = 5e-3


class Cache8:
    """Random 8-bit pages, their values in fp64 and everything that a call needs.  form: "rotary", "plain" or "absorbed"."""

    def __init__(self, form, ctx, h_q=32, h_kv=8, d=128, r_k=512, r_v=512, seed=0, base=500000.0, scale=0.0, amp_k=1.0, amp_v=1.0, unmapped=(), extra=2):
        import torch
        import paper_2410_03111_amd as L
        self.L, self.torch, self.form, self.ctx = L, torch, form, list(ctx)
        rng = np.random.default_rng(seed)
        n = h_kv * d
        if form == "plain":
            r_k = r_v = n
        self.h_q, self.h_kv, self.d, self.base = h_q, h_kv, d, base
        self.scale = scale or d ** -0.5
        self.desc = L.layer_desc(64, h_q, h_kv, d, r_k, r_v, base, scale)
        b = len(self.ctx)
        self.max_pages = max(1, max(-(-c // PAGE) for c in self.ctx)) + 1
        self.n_pages = b * self.max_pages + extra
        self.table = gen.block_table(b, self.max_pages, self.n_pages, seed=seed + 1)
        spec = np.ones(r_k) if form == "plain" else gen.power_law_spectrum(n)[:r_k]
        spec_v = np.ones(r_v) if form == "plain" else gen.power_law_spectrum(n)[:r_v]
        idx = page_gather_indices(r_k, r_v)
        pool = np.full((self.n_pages, co.page_size(r_k, r_v)), 0x7F, np.uint8)       # NaN codes where nothing is cached
        pool[:, PAGE * (r_k + r_v):] = 0xFF
        self.C_k, self.C_v = [], []
        for s, N in enumerate(self.ctx):
            parts = []
            for part, r, sp, amp in ((False, r_k, spec, amp_k), (True, r_v, spec_v, amp_v)):
                amps = amp(rng, N) if callable(amp) else amp
                codes, k = co.quantize(gen.bf16_round((rng.standard_normal((N, r)) * sp * amps).astype(np.float32)))
                for p in range(-(-N // PAGE)):
                    rows = slice(p * PAGE, min(N, p * PAGE + PAGE))
                    cnt = rows.stop - rows.start
                    cols = idx[:cnt, :r_k] if not part else idx[:cnt, r_k:]
                    page = pool[self.table[s, p]]
                    page[cols] = codes[rows]
                    for g in range(k.shape[1]):
                        page[co.scale_index(r_k, r_v, 0, 128 * g, part) + np.arange(cnt)] = (k[rows, g] + 127).astype(np.uint8)
                parts.append(co.dequantize(codes, k))
            for s2, p in unmapped:
                if s2 == s:
                    for x in parts:
                        x[p * PAGE:(p + 1) * PAGE] = 0.0
            self.C_k.append(parts[0])
            self.C_v.append(parts[1])
        for i, (s, p) in enumerate(unmapped):
            self.table[s, p] = (-1, self.n_pages, -2 ** 31, 2 ** 31 - 1)[i % 4]
        self.B_k, self.B_v = (gen.bf16_round((rng.standard_normal((r, n)) / np.sqrt(n)).astype(np.float32)) for r in (r_k, r_v))
        self.q = gen.bf16_round(rng.standard_normal((b, h_q, d)).astype(np.float32))
        bf = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(torch.bfloat16).contiguous()  # noqa: E731
        self.i32 = lambda v: torch.as_tensor(np.ascontiguousarray(v, np.int32)).cuda()  # noqa: E731
        B = (None, None) if form == "plain" else (bf(self.B_k), bf(self.B_v))
        if form == "absorbed":
            per_head = self.B_k.reshape(r_k, h_kv, d)
            self.q = gen.bf16_round(np.stack([[per_head[:, h // (h_q // h_kv)] @ self.q[s, h] for h in range(h_q)] for s in range(b)]).astype(np.float32))
        self.packed = L.pack_factors(self.desc, bf(np.zeros((64, r_k))), bf(np.zeros((64, r_v))), *B)
        self.pool, self.block_table, self.dq = torch.from_numpy(pool.reshape(-1)).cuda(), self.i32(self.table), bf(self.q)
        self.size = {"rotary": L.decode_quantized_workspace_bytes, "plain": L.decode_plain_quantized_workspace_bytes,
                     "absorbed": L.decode_absorbed_quantized_workspace_bytes}[form]

    def call(self, q_pos=None, max_ctx=None, **kw):
        L = self.L
        max_ctx = max(self.ctx) if max_ctx is None else max_ctx
        q_pos = [max(c - 1, 0) for c in self.ctx] if q_pos is None else q_pos
        tail = (self.i32(self.ctx), max_ctx, self.packed, self.pool, self.block_table)
        if self.form == "absorbed":
            return L.decode_attention_absorbed_quantized(self.desc, self.dq, *tail, **kw)
        fn = L.decode_attention_plain_quantized if self.form == "plain" else L.decode_attention_quantized
        return fn(self.desc, self.dq, self.i32(q_pos), *tail, **kw)

    def oracle(self, q_pos=None, max_ctx=None):
        out, G = np.zeros((len(self.ctx), self.h_q, self.d)), self.h_q // self.h_kv
        for s, N in enumerate(self.ctx):
            N = min(N, max(self.ctx) if max_ctx is None else max_ctx)
            if N <= 0:
                continue
            C_k, C_v = self.C_k[s][:N], self.C_v[s][:N]
            V = orc.split_heads(C_v if self.form == "plain" else C_v @ self.B_v.astype(np.float64), self.h_kv, self.d)
            if self.form == "absorbed":
                for h in range(self.h_q):
                    w = orc.softmax_rows((C_k @ self.q[s, h].astype(np.float64) * self.scale)[None])[0]
                    out[s, h] = w @ (C_v @ self.B_v.astype(np.float64))[:, h // G * self.d:(h // G + 1) * self.d]
            else:
                K = orc.split_heads(C_k if self.form == "plain" else C_k @ self.B_k.astype(np.float64), self.h_kv, self.d)
                out[s] = orc.attention_decode(self.q[s].astype(np.float64), self.ctx[s] - 1 if q_pos is None else q_pos[s], K, V, np.arange(N), self.base, self.scale)
        return out

    def check(self, got=None, **kw):
        got = (self.call(**kw) if got is None else got).float().cpu().numpy().astype(np.float64)
        ref = self.oracle(**kw)
        assert np.all(np.isfinite(got))
        n2, mx = np.linalg.norm(got - ref) / np.linalg.norm(ref), np.abs(got - ref).max() / np.abs(ref).max()
        assert n2 <= NORM2 and mx <= TOL, (n2, mx)
        for s, N in enumerate(self.ctx):
            if N == 0:
                assert np.all(got[s] == 0.0)
        return got


LENGTHS = [1, 0, 31, 32, 33, 63, 64, 65, 127, 500]
SHAPES = {
    "plain 8b": dict(form="plain"),
    "plain one head": dict(form="plain", h_q=1, h_kv=1),
    "plain 3 kv heads": dict(form="plain", h_q=21, h_kv=3),
    "plain wide group": dict(form="plain", h_q=32, h_kv=1),
    "plain groups of 20": dict(form="plain", h_q=60, h_kv=3),
    "plain 64 heads": dict(form="plain", h_q=64, h_kv=16),
    "plain 40 kv heads": dict(form="plain", h_q=40, h_kv=40),
    "absorbed 8b": dict(form="absorbed"),
    "absorbed small": dict(form="absorbed", h_q=4, h_kv=2, d=64, r_k=32, r_v=32),
    "absorbed uneven": dict(form="absorbed", h_q=7, h_kv=7, r_k=160, r_v=96),
    "absorbed 64 heads": dict(form="absorbed", h_q=64, h_kv=8, r_k=384, r_v=288),
    "absorbed 40 heads": dict(form="absorbed", h_q=40, h_kv=8, r_k=288, r_v=512),
    "absorbed rank 1024": dict(form="absorbed", h_q=16, h_kv=8, r_k=1024, r_v=1024),
    "absorbed wide keys": dict(form="absorbed", r_k=800, r_v=64),
    "absorbed wide values": dict(form="absorbed", r_k=64, r_v=544),
    "rotary 8b": dict(form="rotary"),
    "rotary 70b": dict(form="rotary", h_q=64, h_kv=8),
    "rotary tiny": dict(form="rotary", h_q=4, h_kv=2, d=64, r_k=32, r_v=32),
    "rotary d 64": dict(form="rotary", h_q=24, h_kv=8, d=64, r_k=288, r_v=224),
    "rotary uneven": dict(form="rotary", h_q=6, h_kv=2, r_k=96, r_v=160),
    "rotary uneven wide": dict(form="rotary", h_q=12, h_kv=4, r_k=448, r_v=64),
    "rotary narrow keys": dict(form="rotary", r_k=128, r_v=512),
    "rotary odd kv heads": dict(form="rotary", h_q=15, h_kv=5, r_k=320, r_v=352),
    "rotary groups of 16": dict(form="rotary", h_q=32, h_kv=2, r_k=256, r_v=256),
    "rotary group of 32": dict(form="rotary", h_q=32, h_kv=1, r_k=64, r_v=128),
    "rotary groups of 8": dict(form="rotary", h_q=64, h_kv=8, r_k=480, r_v=416),
    "rotary groups of 1": dict(form="rotary", h_q=16, h_kv=16, r_k=192, r_v=512),
    "rotary rank 1024": dict(form="rotary", r_k=1024, r_v=1024),
    "rotary wide values": dict(form="rotary", r_k=256, r_v=768),
    "rotary rank 576": dict(form="rotary", r_k=576, r_v=576),
    "rotary rank 768, 64 heads": dict(form="rotary", h_q=64, h_kv=8, r_k=768, r_v=736),
    "rotary wide keys": dict(form="rotary", h_q=24, h_kv=12, r_k=800, r_v=96),
    "rotary groups of 12": dict(form="rotary", h_q=60, h_kv=5, r_k=416, r_v=448),
    "rotary group of 20": dict(form="rotary", h_q=40, h_kv=2, r_k=224, r_v=32),
    "rotary d 64, groups of 5, odd kv heads": dict(form="rotary", h_q=15, h_kv=3, d=64, r_k=128, r_v=96),
    "rotary d 64, groups of 12": dict(form="rotary", h_q=24, h_kv=2, d=64, r_k=64, r_v=128),
    "rotary d 64, one group of 32": dict(form="rotary", h_q=32, h_kv=1, d=64, r_k=64, r_v=64),
    "rotary d 64, one head": dict(form="rotary", h_q=1, h_kv=1, d=64, r_k=64, r_v=32),
    "rotary d 64, rank 1024": dict(form="rotary", h_q=32, h_kv=16, d=64, r_k=1024, r_v=992),
    "rotary d 64, rank 608": dict(form="rotary", h_q=20, h_kv=10, d=64, r_k=608, r_v=576),
}


@pytest.mark.parametrize("name", SHAPES)
def test_lengths(name):
    Cache8(ctx=LENGTHS, **SHAPES[name]).check()


@pytest.mark.parametrize("name", ["plain 8b", "plain groups of 20", "absorbed 8b", "absorbed 64 heads", "rotary 8b", "rotary 70b", "rotary uneven", "rotary rank 1024", "rotary rank 768, 64 heads", "rotary groups of 12",
                                  "rotary d 64", "rotary d 64, groups of 5, odd kv heads", "absorbed rank 1024"])
@pytest.mark.parametrize("ctx", [[3001], [1, 2500, 700, 1337]])
def test_longer_contexts(name, ctx):
    Cache8(ctx=ctx, seed=11, **SHAPES[name]).check()


FORMS = {"plain": dict(form="plain", h_q=8, h_kv=2), "absorbed": dict(form="absorbed", h_q=8, h_kv=2, r_k=160, r_v=128),
         "absorbed wide": dict(form="absorbed", h_q=10, h_kv=5, r_k=64, r_v=544),
         "rotary": dict(form="rotary", h_q=8, h_kv=2, r_k=192, r_v=256), "rotary wide": dict(form="rotary", h_q=24, h_kv=2, r_k=160, r_v=192), "rotary d 64": dict(form="rotary", h_q=6, h_kv=3, d=64, r_k=64, r_v=96)}


@pytest.mark.parametrize("name", FORMS)
def test_pages_that_are_not_mapped_count_as_zeros(name):
    Cache8(ctx=[300, 64, 129, 200], unmapped=[(0, 1), (1, 0), (2, 2), (0, 4), (3, 3)], seed=2, **FORMS[name]).check()


@pytest.mark.parametrize("name", FORMS)
def test_nothing_mapped_gives_zeros(name):
    c = Cache8(ctx=[100, 64], unmapped=[(0, 0), (0, 1), (1, 0)], seed=3, **FORMS[name])
    assert np.all(c.call().float().cpu().numpy() == 0.0)


@pytest.mark.parametrize("name", FORMS)
def test_only_empty_sequences(name):
    c = Cache8(ctx=[0, 0], seed=4, **FORMS[name])
    assert np.all(c.call().float().cpu().numpy() == 0.0)


@pytest.mark.parametrize("name", FORMS)
def test_lengths_beyond_max_ctx_are_clamped(name):
    Cache8(ctx=[300, 64, 150], seed=5, **FORMS[name]).check(max_ctx=140)


def uneven(low, high):
    return lambda rng, n: 2.0 ** rng.integers(low, high + 1, (n, 1))


@pytest.mark.parametrize("name", FORMS)
def test_values_whose_scales_differ_from_position_to_position(name):
    Cache8(ctx=[333, 70], amp_v=uneven(-8, 3), seed=6, **FORMS[name]).check()


@pytest.mark.parametrize("name", FORMS)
def test_values_that_are_zero_at_some_positions(name):
    Cache8(ctx=[200, 90], amp_v=lambda rng, n: (rng.random((n, 1)) < 0.5) * 1.0, seed=7, **FORMS[name]).check()


@pytest.mark.parametrize("name", FORMS)
def test_a_heavy_position_of_small_values(name):
    """One position takes most of the weight, its values are 2^-9 of the others'."""
    c = Cache8(ctx=[150], amp_v=lambda rng, n: np.where(np.arange(n)[:, None] == 40, 2.0 ** -9, 1.0),
               amp_k=lambda rng, n: np.where(np.arange(n)[:, None] == 40, 4.0, 0.1), seed=8, **FORMS[name])
    c.check()


@pytest.mark.parametrize("name", FORMS)
def test_all_values_zero(name):
    c = Cache8(ctx=[130], amp_v=0.0, seed=9, **FORMS[name])
    assert np.all(c.call().float().cpu().numpy() == 0.0)


@pytest.mark.parametrize("name", FORMS)
def test_a_nan_in_the_cache_reaches_its_sequence_only(name):
    c = Cache8(ctx=[100, 80], seed=10, **FORMS[name])
    page = int(c.table[0, 1])
    pool = c.pool.view(c.n_pages, -1)
    pool[page, int(page_gather_indices(c.desc.rank_k, c.desc.rank_v)[3, 0])] = 0x7F
    got = c.call().float().cpu().numpy()
    assert np.isnan(got[0]).any() and np.isfinite(got[1]).all()


@pytest.mark.parametrize("name", FORMS)
def test_far_positions_and_queries_elsewhere(name):
    if name != "absorbed":
        Cache8(ctx=[400, 33], seed=12, **FORMS[name]).check(q_pos=[100000, 0])


@pytest.mark.parametrize("name", FORMS)
def test_softmax_scale_of_the_layer(name):
    Cache8(ctx=[150, 40], scale=0.05, seed=13, **FORMS[name]).check()


@pytest.mark.parametrize("name", FORMS)
def test_a_workspace_of_another_call_and_one_split(name):
    import torch
    c = Cache8(ctx=[900, 500], seed=14, **FORMS[name])
    whole = c.check()
    big = c.size(c.desc, 16, 100000)
    again = c.call(workspace=torch.empty(big, dtype=torch.uint8, device="cuda"))
    assert np.array_equal(again.float().cpu().numpy(), whole)
    width = 128 if c.form == "plain" else c.desc.rank_v
    one = -(-2 * c.h_q * 8 // 256) * 256 + -(-2 * c.h_q * width * 2 // 256) * 256
    c.check(got=c.call(workspace=torch.empty(one, dtype=torch.uint8, device="cuda")))
    with pytest.raises(c.L.LorcError) as e:
        c.call(workspace=torch.empty(one - 256, dtype=torch.uint8, device="cuda"))
    assert e.value.code == c.L.EWORKSPACE


@pytest.mark.parametrize("name", FORMS)
def test_pools_beyond_4_gib(name):
    import torch
    c = Cache8(ctx=[130], seed=15, **FORMS[name])
    want = c.call().float().cpu().numpy()
    size = c.L.page_bytes_quantized(c.desc)
    n = (5 << 30) // size
    pool = torch.zeros(n, size, dtype=torch.uint8, device="cuda")
    far = n - 1 - np.arange(c.max_pages)
    for p in range(c.max_pages):
        pool[int(far[p])] = c.pool.view(c.n_pages, size)[int(c.table[0, p])]
    c.pool, c.block_table = pool, c.i32(far[None])
    assert np.array_equal(c.call().float().cpu().numpy(), want)


@pytest.mark.parametrize("name", FORMS)
def test_replays_from_a_graph_on_another_stream(name):
    import torch
    c = Cache8(ctx=[700, 129, 64], seed=16, **FORMS[name])
    out, ws = torch.zeros(3, c.h_q, c.d, dtype=torch.bfloat16, device="cuda"), torch.empty(c.size(c.desc, 3, 700), dtype=torch.uint8, device="cuda")
    ctx, q_pos = c.i32(c.ctx), c.i32([n - 1 for n in c.ctx])

    def step():
        if c.form == "absorbed":
            c.L.decode_attention_absorbed_quantized(c.desc, c.dq, ctx, 700, c.packed, c.pool, c.block_table, out=out, workspace=ws)
        else:
            fn = c.L.decode_attention_plain_quantized if c.form == "plain" else c.L.decode_attention_quantized
            fn(c.desc, c.dq, q_pos, ctx, 700, c.packed, c.pool, c.block_table, out=out, workspace=ws)

    step()
    c.check(got=out)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.current_stream().wait_stream(side)
    for rep in range(4):
        c.dq.copy_(torch.randn(c.dq.shape, device="cuda").to(torch.bfloat16))
        out.fill_(float("nan"))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        step()
        torch.cuda.synchronize()
        assert torch.equal(got, out) and bool(torch.isfinite(got).all()), rep


@pytest.mark.parametrize("name", FORMS)
def test_short_sequences_whose_pages_come_from_memory(name):
    """The one page of a sequence is asked for and used within a few hundred cycles: nothing may be read before it has landed.  Between the
    calls the caches are filled with something else, and LDS with the scales of much larger values."""
    import torch
    c = Cache8(ctx=[1 + 3 * s % 64 for s in range(96)], seed=19, **FORMS[name])
    other = Cache8(ctx=[200, 64, 130], seed=20, amp_v=2.0 ** 40, **FORMS[name])
    other.block_table, other.ctx = other.block_table.repeat(32, 1), other.ctx * 32
    other.dq = other.dq.repeat(32, 1, 1)
    want = c.call()
    c.check(got=want)
    large = torch.empty(3 << 28, dtype=torch.uint8, device="cuda")
    for rep in range(12):
        other.call()
        large.fill_(rep)
        assert torch.equal(c.call(), want), rep


@pytest.mark.parametrize("name", ["plain", "absorbed", "rotary"])
def test_rows_of_the_table_behind_the_batch_and_refused_arguments(name):
    import torch
    c = Cache8(ctx=[70, 130], seed=17, **FORMS[name])
    L = c.L
    want = c.call()
    out = torch.full((3, c.h_q, c.d), 7.0, dtype=torch.bfloat16, device="cuda")
    c.block_table = torch.cat([c.block_table, torch.full_like(c.block_table[:1], 0)])       # a third row that no sequence has
    c.call(out=out[:2])
    assert torch.equal(out[:2], want) and bool((out[2] == 7.0).all())
    fn = {"plain": L.decode_attention_plain_quantized, "absorbed": L.decode_attention_absorbed_quantized, "rotary": L.decode_attention_quantized}[name]
    ctx, pos = c.i32(c.ctx), c.i32([69, 129])
    q, first = ("q_lat", {}) if name == "absorbed" else ("q", dict(q_pos=pos))
    good = {"desc": c.desc, q: c.dq, **first, "ctx_len": ctx, "max_ctx": 130, "packed": c.packed, "cache_q8": c.pool, "block_table": c.block_table}
    assert torch.equal(fn(**good), want)
    bad = [(q, c.dq.float(), TypeError), (q, c.dq[:, ::2], TypeError), (q, c.dq[:, :1].contiguous(), ValueError), ("ctx_len", ctx[:1], ValueError),
           ("ctx_len", ctx.to(torch.int64), TypeError), ("packed", c.packed[:64], ValueError), ("packed", c.packed.cpu(), TypeError), ("cache_q8", c.pool[:10], L.LorcError),
           ("block_table", c.block_table[:1], ValueError), ("block_table", c.block_table[:, ::2], TypeError), ("max_ctx", 10 ** 6, L.LorcError), ("max_ctx", -1, L.LorcError),
           ("out", out, ValueError), ("out", out[:2].float(), TypeError), ("workspace", torch.zeros(64, dtype=torch.uint8, device="cuda"), L.LorcError)]
    if first:
        bad += [("q_pos", pos[:1], ValueError), ("q_pos", pos.cpu(), TypeError)]
    for key, value, error in bad:
        with pytest.raises(error):
            fn(**{**good, key: value})


@pytest.mark.parametrize("name", FORMS)
def test_a_query_of_nan_stays_in_its_head(name):
    c = Cache8(ctx=[300, 65], seed=18, **FORMS[name])
    want = c.call().float().cpu().numpy()
    c.dq[0, 1] = float("nan")
    got = c.call().float().cpu().numpy()
    assert np.all(np.isnan(got[0, 1]))
    got[0, 1] = want[0, 1]
    assert np.array_equal(got, want)


def test_a_served_prompt_from_prefill_to_its_forks():
    """Append, prefill, into the 8-bit cache, three answers that share the prompt's pages, decode steps of their own, a finished one
    released, the pool made dense under the others: every step against fp64 on the values that the pages stand for."""
    import torch
    import paper_2410_03111_amd as L
    rng = np.random.default_rng(20)
    D, h_q, h_kv, d, r = 256, 8, 2, 128, 192
    n, N = h_kv * d, 150
    desc = L.layer_desc(D, h_q, h_kv, d, r, r, 10000.0)
    bf = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.float32)).cuda().to(torch.bfloat16).contiguous()  # noqa: E731
    i32 = lambda v: torch.as_tensor(np.ascontiguousarray(v, np.int32)).cuda()  # noqa: E731
    A = [bf(rng.standard_normal((D, r)) / 16) for _ in range(2)]
    B = [bf(rng.standard_normal((r, n)) / 16) for _ in range(2)]
    packed = L.pack_factors(desc, *A, *B)
    n_pages, max_pages = 24, 5
    table, refs = i32(np.full((4, max_pages), -1)), i32(np.zeros(n_pages))
    pool = torch.full((n_pages, L.page_bytes_quantized(desc)), 0x7F, dtype=torch.uint8, device="cuda")
    # the bf16 side: a prompt's pages, later one page per sequence that every page of positions reuses
    prompt_table = i32(np.arange(4 * max_pages).reshape(4, max_pages))
    open_table = i32(np.repeat(np.arange(4)[:, None], max_pages, 1))
    cache = torch.zeros(4 * max_pages, L.page_bytes(desc), dtype=torch.uint8, device="cuda")

    blocker = i32([3])
    L.reserve_pages(table, refs, blocker, i32([200]), i32([0]))               # pages that are freed below: the pool gets a hole
    x = bf(rng.standard_normal((N, D)))
    L.append_latent(desc, x, packed, i32(np.zeros(N)), i32(np.arange(N)), prompt_table, cache)
    out = L.prefill_attention(desc, bf(rng.standard_normal((N, h_q, d))), i32([0, N]), N, packed, cache, prompt_table)
    assert bool(torch.isfinite(out).all())
    status = i32([9])
    L.reserve_pages(table, refs, i32([0]), i32([N]), status)
    L.quantize_latents(desc, cache, prompt_table, i32([0]), i32([N]), N, pool, table)
    src, dst, st2 = (i32([0, 0]) for _ in range(3))
    L.fork_sequences(table, refs, i32([0, 0]), i32([1, 2]), i32([N, N]), src, dst, st2)
    L.copy_pages(pool, src, dst)
    assert status.tolist() == [0] and st2.tolist() == [0, 0]
    t = table.cpu().numpy()
    assert t[1, :2].tolist() == t[0, :2].tolist() == t[2, :2].tolist() and len({t[s, 2] for s in range(3)}) == 3

    idx = page_gather_indices(r, r)

    def values(s, length):
        pg, tb = pool.cpu().numpy(), table.cpu().numpy()
        rows = []
        for pos in range(length):
            page = pg[tb[s, pos // PAGE]]
            k = [int(page[co.scale_index(r, r, pos % PAGE, 128 * g, part)]) - 127 for part in (False, True) for g in range(2)]
            c = page[idx[pos % PAGE]]
            rows.append(np.concatenate([co.dequantize(c[:r], np.array(k[:2])), co.dequantize(c[r:], np.array(k[2:]))]))
        return np.array(rows)

    Bk, Bv = (b.float().cpu().numpy().astype(np.float64) for b in B)
    lens, live = [N, N, N], [0, 1, 2]

    def step(live):
        seqs = i32(live)
        pos = [lens[s] for s in live]
        for s in live:
            lens[s] += 1
        st = i32(np.full(len(live), 9))
        L.reserve_pages(table, refs, seqs, i32([lens[s] for s in live]), st)
        assert st.tolist() == [0] * len(live)
        L.append_latent(desc, bf(rng.standard_normal((len(live), D))), packed, seqs, i32(pos), open_table, cache)
        rows, opens = table[live].contiguous(), open_table[live].contiguous()
        L.quantize_latents(desc, cache, opens, i32(pos), i32([p + 1 for p in pos]), 1, pool, rows)
        q = gen.bf16_round(rng.standard_normal((len(live), h_q, d)).astype(np.float32))
        got = L.decode_attention_quantized(desc, bf(q), i32(pos), i32([p + 1 for p in pos]), max(pos) + 1, packed, pool, rows).float().cpu().numpy().astype(np.float64)
        for i, s in enumerate(live):
            c = values(s, lens[s])
            ref = orc.attention_decode(q[i].astype(np.float64), pos[i], orc.split_heads(c[:, :r] @ Bk, h_kv, d), orc.split_heads(c[:, r:] @ Bv, h_kv, d),
                                       np.arange(lens[s]), 10000.0)
            assert np.linalg.norm(got[i] - ref) / np.linalg.norm(ref) <= NORM2

    shared = values(0, 128)
    for _ in range(3):
        step(live)
    L.free_sequences(table, refs, i32([1, 3]))
    before = [values(s, lens[s]) for s in (0, 2)]
    msrc, mdst, new = i32(np.zeros(12)), i32(np.zeros(12)), i32(np.zeros(n_pages))
    L.compact_pages(table, refs, msrc, mdst, new)
    L.copy_pages(pool, msrc, mdst)
    assert int((msrc >= 0).sum()) > 0
    for s, want in zip((0, 2), before):
        assert np.array_equal(values(s, lens[s]), want)
    assert np.array_equal(values(2, 128), shared)
    step([0, 2])
    used = refs.cpu().numpy() > 0
    L.free_sequences(table, refs, i32([0, 2]))
    assert used.sum() == 4 and int(refs.sum()) == 0 and int((table >= 0).sum()) == 0
