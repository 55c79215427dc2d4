"""Attention over an 8-bit pool against the formula in 64 bits, on the values the pool's read returns."""
import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
from q8_util import TORCH, attend, attend_rule, context_for, held, model, offsets, pool_for, seen_by_rows, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Case:
    """Entries of the given lengths in layer 1 of 2, their cached values in 64 bits, and a context."""

    def __init__(self, d, heads, dtype, form, lens, rows, seed=0, spread=0.6, check=None):
        self.d, self.heads, self.dtype, self.form, self.lens, self.rows = d, heads, dtype, form, lens, rows
        m = model(d, heads, dtype, form)
        self.rng = np.random.default_rng(seed)
        self.ctx = context_for(m, len(lens), max(1, sum(rows)))
        self.pool, self.handles = pool_for(self.ctx.cfg, dtype, lens)
        (k, k64), (v, v64) = (values(self.rng, sum(lens), d, dtype, spread) for _ in range(2))
        rg.relaygr_kv_pool_write(self.pool, 1, rg.KvRows(self.handles, offsets(lens)), k.to(DEV), v.to(DEV))
        at = offsets(lens)
        self.checked = range(len(lens)) if check is None else check
        self.k, self.v = ([None if u not in self.checked else held(x[at[u]:at[u + 1]].reshape(n, heads, d // heads), dtype) for u, n in enumerate(lens)] for x in (k64, v64))
        self.q, self.q64 = values(self.rng, sum(rows), d, dtype, spread)
        self.q = self.q.to(DEV)

    def run(self, key_len=None, causal=False, **kw):
        rows = rg.KvRows(self.handles, offsets(self.rows), key_len=key_len)
        return rg.relaygr_cache_attend(self.ctx, self.pool, 1, rows, kw.pop("q", self.q), causal=causal, **kw)

    def check(self, out, key_len=None, causal=False, users=None):
        got = out.double().cpu().numpy()
        ro = offsets(self.rows)
        for u in range(len(self.lens)) if users is None else users:
            n, m = self.lens[u] if key_len is None else key_len[u], self.rows[u]
            q = self.q64[ro[u]:ro[u + 1]].reshape(m, self.heads, self.d // self.heads)
            want, bound = attend(q, self.k[u][:n], self.v[u][:n], seen_by_rows(n, m, causal), self.form, self.dtype)
            g = got[ro[u]:ro[u + 1]].reshape(want.shape)
            assert np.isfinite(g).all(), u
            off = np.abs(g - want) / bound
            assert off.max(initial=0.0) <= 1.0, f"user {u} ({m} rows, {n} keys): {off.max():.2f} of the bound at {np.unravel_index(off.argmax(), off.shape)}"


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,heads", [(128, 4), (256, 4), (256, 8), (512, 8), (512, 4), (1024, 8), (128, 1)])
def test_ragged_batches(d, heads, dtype, form):
    """Histories that end before, at and behind a block's end, rows of one to a few row tiles."""
    lens = [1, 64, 65, 200, 63, 700, 129, 2]
    rows = [1, 3, 33, 64, 65, 31, 0, 130]
    c = Case(d, heads, dtype, form, lens, rows, seed=d)
    c.check(c.run())


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("rows", [1, 2, 17, 32, 33, 64, 70, 257])
def test_row_counts(form, rows):
    lens = [500, 20]
    c = Case(256, 4, "bf16", form, lens, [rows, rows], seed=rows)
    c.check(c.run())
    c.check(c.run(causal=True), causal=True)


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("d,heads,dtype", [(256, 8, "fp16"), (256, 4, "bf16"), (512, 4, "fp16")])
def test_causal_rows_and_rows_that_see_nothing(d, heads, dtype, form):
    """Appended rows see up to their own token; with more rows than keys the first see nothing, as do all where key_len is 0."""
    lens, rows, key_len = [300, 64, 200, 10, 90], [100, 64, 65, 40, 7], [300, 64, 130, 10, 0]
    c = Case(d, heads, dtype, form, lens, rows, seed=3)
    out = c.run(key_len=key_len, causal=True)
    c.check(out, key_len=key_len, causal=True)
    ro = offsets(rows)
    assert not out[ro[3]:ro[3] + 30].any() and not out[ro[4]:].any()
    c.check(c.run(key_len=key_len), key_len=key_len)


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("lens,rows", [([5000], [1]), ([16384], [5]), ([3000, 100, 9000], [1, 40, 2]), ([4100], [300])])
def test_long_histories_cut_along_the_keys(lens, rows, form):
    c = Case(256, 4, "bf16", form, lens, rows, seed=17)
    out = c.run()
    c.check(out)
    # and uncut, where the scratch holds no partial sums: a context of one row
    small = context_for(model(256, 4, "bf16", form), 1, 1)
    ro = rg.KvRows(c.handles, offsets(rows))
    c.check(rg.relaygr_cache_attend(small, c.pool, 1, ro, c.q))
    assert torch.equal(out, c.run())        # the same bits every time


def test_many_users_more_than_a_launch_takes():
    rng = np.random.default_rng(23)
    users = 150
    lens, rows = [int(n) for n in rng.integers(1, 300, users)], [int(n) for n in rng.integers(0, 6, users)]
    c = Case(128, 2, "bf16", "softmax", lens, rows, seed=29)
    c.check(c.run())
    c.check(c.run(causal=True), causal=True)


#   users, rows, keys, d, heads, and what the launch takes: blocks, once, whether it is cut
KERNELS = [
    (33, 200, 70, 512, 8, 2, 0, False),
    (33, 250, [64] * 30 + [700] * 3, 512, 8, 2, 0, True),
    (80, 3, 2100, 512, 8, 1, 1, False),
    (20, 5, [200] * 19 + [9000], 256, 4, 1, 0, True),
    (65, 7, [1100] * 64 + [17000], 1024, 8, 1, 1, True),
]


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("case", range(len(KERNELS)))
def test_the_kernels_of_large_launches(case, form):
    """Items of two row blocks, codes loaded once, launches of many users whose rows are joined: some of the users against the formula."""
    users, m, n, d, heads, blocks, once, cut = KERNELS[case]
    lens = n if isinstance(n, list) else [n] * users
    rows = [m - u % 3 for u in range(users)]
    rule = attend_rule(rows, lens, heads, d // heads)
    assert (rule["blocks"], rule["once"], rule["parts"] > 1) == (blocks, once, cut)
    c = Case(d, heads, "bf16", form, lens, rows, seed=61 + case, check=(0, users // 2, users - 1))
    c.check(c.run(), users=c.checked)
    if blocks == 2:
        c.check(c.run(causal=True), causal=True, users=c.checked)


def test_large_scores():
    """Softmax weights that are nearly one key's alone, scores of hundreds; SiLU of large negative scores."""
    for form in ("softmax", "silu"):
        c = Case(256, 4, "bf16", form, [300, 90], [40, 5], seed=31, spread=1.5)
        c.q.mul_(8.0)
        c.q64 = c.q.double().cpu().numpy()
        c.q.mul_(-1.0)
        c.q64 = -c.q64
        c.check(c.run())


def test_columns_of_wider_arrays_and_neighbours_left_alone():
    c = Case(256, 4, "fp16", "silu", [130, 70], [3, 34], seed=37)
    n, d = sum(c.rows), c.d
    fused = torch.zeros(n, 4 * d, dtype=TORCH[c.dtype], device=DEV)
    fused[:, 2 * d:3 * d] = c.q
    out = torch.full((n + 2, d + 16), 5.0, dtype=TORCH[c.dtype], device=DEV)
    got = c.run(q=fused[:, 2 * d:3 * d].view(n, c.heads, d // c.heads), out=out[1:-1, 8:-8])
    c.check(got)
    assert torch.equal(got, c.run())
    out[1:-1, 8:-8] = 5.0
    assert bool((out == 5.0).all())


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("d,heads,dtype", [(256, 4, "bf16"), (128, 4, "fp16"), (256, 2, "fp16")])
def test_nan_reaches_the_rows_that_see_it_only(d, heads, dtype, form):
    """NaN in K or V of one token of one head: rows before it, other heads and (for V) other features stay as they are."""
    n, m, at, dh = 150, 100, 140, d // heads
    for what in "kv":
        c = Case(d, heads, dtype, form, [n], [m], seed=41)
        k, v = (torch.from_numpy(x[0]).to(TORCH[dtype]).to(DEV).view(n, d) for x in (c.k, c.v))
        clean = c.run(causal=True), c.run(key_len=[at])
        (k if what == "k" else v)[at, dh + 5] = float("nan")
        rg.relaygr_kv_pool_write(c.pool, 1, rg.KvRows(c.handles, [0, n]), k, v)
        # (the block's other values are as before: a NaN does not move its scale unless it stood where the largest did)
        poisoned = c.run(causal=True)
        assert torch.equal(c.run(key_len=[at]), clean[1]), "no row sees the token"
        sees = torch.from_numpy(seen_by_rows(n, m, True) > at)
        bad = torch.isnan(poisoned).view(m, heads, dh).cpu()
        cols = torch.zeros(heads, dh, dtype=torch.bool)
        if what == "k":
            cols[1] = True
        else:
            cols[1, 5] = True
        assert torch.equal(bad, sees[:, None, None] & cols[None])
        assert torch.equal(poisoned.view(m, heads, dh)[:, 2:], clean[0].view(m, heads, dh)[:, 2:])


def test_write_then_attend_token_by_token():
    """A history that grows: each new token is written and then attends over everything up to itself; two graphs of one step too."""
    d, heads, dtype = 256, 4, "bf16"
    c = Case(d, heads, dtype, "softmax", [200, 140], [1, 1], seed=43)
    for step in range(3):
        pos = [100 + step, 63 + step]
        (k, k64), (v, v64) = (values(c.rng, 2, d, dtype) for _ in range(2))
        rg.relaygr_kv_pool_write(c.pool, 1, rg.KvRows(c.handles, [0, 1, 2], first_token=pos), k.to(DEV), v.to(DEV))
        for u, p in enumerate(pos):
            for x, new in ((c.k, k64), (c.v, v64)):
                b0 = p // 64 * 64
                blk = held(np.concatenate([x[u][b0:p], new[u].reshape(1, heads, d // heads)]), dtype)
                x[u][b0:p + 1] = blk
                x[u][p + 1:b0 + 64] = 0.0
        keys = [p + 1 for p in pos]
        c.check(c.run(key_len=keys, causal=True), key_len=keys, causal=True)


def test_captured_attention_replays_on_new_rows():
    c = Case(512, 8, "bf16", "silu", [3000, 400], [20, 3], seed=47)
    rows = rg.KvRows(c.handles, offsets(c.rows))
    out = torch.empty_like(c.q)
    want = c.run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rg.relaygr_cache_attend(c.ctx, c.pool, 1, rows, c.q, out=out)
    for _ in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        q, c.q64 = values(c.rng, sum(c.rows), c.d, c.dtype)
        c.q.copy_(q.to(DEV))
        want = c.run()
        torch.cuda.synchronize()
        c.check(want)


def test_two_streams_share_a_context():
    """Calls of one context on two streams follow one another: the second's partial sums do not run into the first's."""
    c = Case(256, 4, "bf16", "softmax", [9000, 7000], [2, 30], seed=53)
    want = c.run()
    c.check(want)
    a, b = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [c.run(stream=s) for _ in range(5) for s in (a, b)]
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)


def test_refusals():
    c = Case(256, 4, "bf16", "silu", [100, 50], [2, 3], seed=59)

    def code(**kw):
        args = dict(ctx=c.ctx, pool=c.pool, layer=1, rows=rg.KvRows(c.handles, offsets(c.rows)), q=c.q) | kw
        out = torch.full((5, 256), 3.0, dtype=torch.bfloat16, device=DEV)
        with pytest.raises(rg.RelayGRError) as e:
            rg.relaygr_cache_attend(args["ctx"], args["pool"], args["layer"], args["rows"], args["q"], out=out)
        torch.cuda.synchronize()
        assert bool((out == 3.0).all())
        return e.value.code
    assert code(layer=2) == rg.RELAYGR_EINVAL and code(layer=-1) == rg.RELAYGR_EINVAL
    assert code(rows=rg.KvRows(c.handles, [0, 2, 5], key_len=[101, 50])) == rg.RELAYGR_EINVAL
    assert code(rows=rg.KvRows(c.handles, [0, 2, 5], key_len=[-1, 50])) == rg.RELAYGR_EINVAL
    assert code(rows=rg.KvRows([c.handles[0], 12345], [0, 2, 5])) == rg.RELAYGR_ENOENT
    assert code(q=c.q.half()) == rg.RELAYGR_EINVAL and code(q=c.q.cpu()) == rg.RELAYGR_EINVAL and code(q=c.q[:4]) == rg.RELAYGR_EINVAL
    odd = torch.zeros(5 * 256 + 8, dtype=torch.bfloat16, device=DEV)[4:4 + 5 * 256].view(5, 256)
    assert code(q=odd) == rg.RELAYGR_EINVAL
    other = context_for(model(512, 8, "bf16"), 1, 8)
    assert code(ctx=other) == rg.RELAYGR_EINVAL
    half = context_for(model(256, 4, "fp16"), 1, 8)
    assert code(ctx=half) == rg.RELAYGR_EINVAL
    p16 = rg.KvPool(c.ctx.cfg, "bf16", 4 * rg.relaygr_kv_pool_bytes_for(c.ctx.cfg, 64, 64), 64)
    h16 = rg.relaygr_kv_pool_alloc(p16, 1, 100)
    assert code(pool=p16, rows=rg.KvRows([h16], [0, 5])) == rg.RELAYGR_EINVAL
    # no users, or no rows: nothing to do
    assert rg.relaygr_cache_attend(c.ctx, c.pool, 0, rg.KvRows([], [0]), c.q[:0]).shape == (0, 256)
    assert rg.relaygr_cache_attend(c.ctx, c.pool, 0, rg.KvRows(c.handles, [0, 0, 0]), c.q[:0]).shape == (0, 256)


def test_entries_beyond_4_gib_of_the_slab():
    """An entry behind more than 2^32 bytes of others, in the last of many layers."""
    d, heads, dtype = 1024, 8, "bf16"
    m = model(d, heads, dtype, "softmax", layers=16)
    ctx = context_for(m, 1, 70)
    tile = rg.relaygr_kv_pool_bytes_for_q8(ctx.cfg, 64, 64)
    before = (1 << 32) // tile + 3
    pool = rg.KvPool(ctx.cfg, dtype, (before + 4) * tile, 64, quantized=True)
    rg.relaygr_kv_pool_alloc(pool, 1, before * 64)
    h = rg.relaygr_kv_pool_alloc(pool, 2, 200)
    assert rg.relaygr_kv_pool_locate(pool, h, 15, 199, 1023)[0] > 1 << 32
    rng = np.random.default_rng(67)
    (k, k64), (v, v64), (q, q64) = (values(rng, n, d, dtype) for n in (200, 200, 70))
    rg.relaygr_kv_pool_write(pool, 15, rg.KvRows([h], [0, 200]), k.to(DEV), v.to(DEV))
    kh, vh = held(k64.reshape(200, heads, -1), dtype), held(v64.reshape(200, heads, -1), dtype)
    for got, want in zip(rg.relaygr_kv_pool_read(pool, 15, rg.KvRows([h], [0, 200])), (kh, vh)):
        assert np.array_equal(got.double().cpu().numpy(), want.reshape(200, d))
    out = rg.relaygr_cache_attend(ctx, pool, 15, rg.KvRows([h], [0, 70]), q.to(DEV))
    want, bound = attend(q64.reshape(70, heads, -1), kh, vh, [200] * 70, "softmax", dtype)
    assert (np.abs(out.double().cpu().numpy().reshape(want.shape) - want) <= bound).all()


def test_calls_of_every_kind_in_turn_on_one_context():
    """Cut calls that join themselves, captured ones that have a launch for it, and rankings, which use the same scratch: each leaves the others' results as they are."""
    c = Case(256, 4, "bf16", "silu", [9000, 500, 64], [3, 20, 2], seed=71)
    one = rg.KvRows(c.handles[:1], [0, 3])
    many = rg.KvRows(c.handles, offsets(c.rows))
    want = rg.relaygr_cache_attend(c.ctx, c.pool, 1, one, c.q[:3]), c.run()
    c.check(want[1])
    outs = torch.empty_like(want[0]), torch.empty_like(want[1])
    graphs = []
    for rows, q, out in ((one, c.q[:3], outs[0]), (many, c.q, outs[1])):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            rg.relaygr_cache_attend(c.ctx, c.pool, 1, rows, q, out=out)
    batch = rg.Batch({"n_users": 1, "user_ids": [7], "prefix_emb": np.zeros((0, 256), np.float32), "prefix_off": [0, 500],
                      "suffix_emb": np.zeros((0, 256), np.float32), "suffix_off": [0, 0],
                      "cand_emb": np.ones((20, 256), np.float32), "cand_off": [0, 20]}, "bf16", handles=[c.handles[1]])
    for turn in range(3):
        for out in outs:
            out.zero_()
        graphs[turn % 2].replay()
        assert torch.equal(c.run(), want[1])
        graphs[1 - turn % 2].replay()
        rg.relaygr_rank_with_cache(c.ctx, c.pool, batch)
        assert torch.equal(rg.relaygr_cache_attend(c.ctx, c.pool, 1, one, c.q[:3]), want[0])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], want[0]) and torch.equal(outs[1], want[1])


def test_one_history_for_many_users_and_a_batch_with_idle_ones():
    """The same entry in several users' places, users without rows between them."""
    c = Case(256, 4, "fp16", "softmax", [300], [40], seed=73)
    h = c.handles[0]
    rows = rg.KvRows([h] * 5, [0, 10, 10, 25, 25, 40], key_len=[300, 5, 300, 300, 300])
    out = rg.relaygr_cache_attend(c.ctx, c.pool, 1, rows, c.q)
    c.check(out)
    k, v = rg.relaygr_kv_pool_read(c.pool, 1, rg.KvRows([h, h], [0, 300, 400], first_token=[0, 100]))
    assert torch.equal(k[300:], k[100:200]) and torch.equal(v[300:], v[100:200])


@pytest.mark.parametrize("form", ["silu", "softmax"])
def test_a_context_with_little_scratch(form):
    """Rows are cut only as far as the scratch holds their partial sums: fewer pieces, or none, and the same answers."""
    d, heads, lens, rows = 128, 1, [16384], [300]
    parts = attend_rule(rows, lens, heads, d // heads)["parts"]
    small = context_for(model(d, heads, "bf16", form), 1, 1)
    weights = 2 * 5 * d * d * 2
    assert parts > 1 and parts * rows[0] * d * 4 > rg.relaygr_scratch_bytes(small.cfg, 1, 0, 1) - weights
    c = Case(d, heads, "bf16", form, lens, rows, seed=83)
    c.check(c.run())
    c.ctx = small
    c.check(c.run())
    c.check(c.run(causal=True), causal=True)
