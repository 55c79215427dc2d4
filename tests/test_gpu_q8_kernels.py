"""Attention over an 8-bit pool: each kernel that a launch's sizes can ask for, in both storage types, calls of different sizes on two streams, contexts
without room for partial sums, and captured steps."""
import ctypes as C
import types

import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
from paper_2601_01712_amd import binding as B
from q8_util import TORCH, attend_rule, context_for, model, offsets, rule_shim, seen_by_rows, values
from test_gpu_q8_attend import Case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FEW = 16          # users of the launches that may join the pieces of their rows themselves


def joins_itself(rows, lens, heads, dh):
    """Whether an eager launch joins its pieces itself; None where it has none to join."""
    rule = attend_rule(rows, lens, heads, dh)
    parts = [rule_shim().attend_parts_of(-(-n // 64), rule["piece"]) for n in lens]
    if max(parts) == 1:
        return None
    if len(rows) > FEW or rule["blocks"] > 1 or rule["once"]:
        return False
    joins = rule_shim().attend_joins
    joins.argtypes = [C.c_int, C.c_int64, C.c_int]
    return bool(joins(max(min(m, 32) * p for m, p in zip(rows, parts)), sum(-(-m // 32) * p for m, p in zip(rows, parts)) * heads, 4096))


LONG_ONE = [200] * 19 + [9000]
#   users, rows, keys, d, heads, storage type, and what the launch takes: blocks, once, whether it is cut
KERNELS = [
    (33, 200, 70, 512, 8, "fp16", 2, 0, False),
    (33, 250, [64] * 30 + [700] * 3, 512, 8, "fp16", 2, 0, True),
    (80, 3, 2100, 512, 8, "fp16", 1, 1, False),
    (65, 7, [1100] * 64 + [17000], 1024, 8, "fp16", 1, 1, True),
    (80, 3, 3300, 256, 8, "bf16", 1, 1, False),                 # d_head 32
    (65, 7, [4100] * 64 + [40000], 256, 8, "fp16", 1, 1, True),
    (20, 5, LONG_ONE, 256, 8, "bf16", 1, 0, True),              # the joins of d_head 32 (eight groups of pieces), 64 and 128
    (20, 5, LONG_ONE, 256, 8, "fp16", 1, 0, True),
    (20, 5, LONG_ONE, 256, 4, "fp16", 1, 0, True),
    (20, 5, LONG_ONE, 256, 2, "fp16", 1, 0, True),
    (20, 5, LONG_ONE, 128, 4, "fp16", 1, 0, True),              # rows of half a wavefront
]


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("case", range(len(KERNELS)))
def test_the_kernels_of_large_launches_in_either_type(case, form):
    users, m, n, d, heads, dtype, blocks, once, cut = KERNELS[case]
    lens = n if isinstance(n, list) else [n] * users
    rows = [m - u % 3 for u in range(users)]
    rule = attend_rule(rows, lens, heads, d // heads)
    assert (rule["blocks"], rule["once"], rule["parts"] > 1) == (blocks, once, cut)
    assert joins_itself(rows, lens, heads, d // heads) is (False if cut else None)
    c = Case(d, heads, dtype, form, lens, rows, seed=161 + case, check=(0, users // 2, users - 1))
    out = c.run()
    c.check(out, users=c.checked)
    assert torch.equal(out, c.run())
    if blocks == 2:
        c.check(c.run(causal=True), causal=True, users=c.checked)


#   rows, keys, d, heads, whether the launch joins itself
FEW_USERS = [
    ([1], [5000], 256, 8, True), ([7, 3], [4100, 300], 256, 8, True), ([300], [4100], 256, 8, True), ([20], [9000], 256, 8, False),
    ([1], [5000], 256, 2, True), ([40], [9000], 256, 2, False), ([2, 2], [3000, 5000], 128, 4, True),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("case", range(len(FEW_USERS)))
def test_either_join_of_few_users(case, form, dtype):
    """Pieces joined by the launch itself and, in a graph, by a second one: the formula, and the same bits."""
    rows, lens, d, heads, itself = FEW_USERS[case]
    assert joins_itself(rows, lens, heads, d // heads) is itself
    c = Case(d, heads, dtype, form, lens, rows, seed=211 + case)
    out = c.run()
    c.check(out)
    replayed = torch.zeros_like(out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.run(out=replayed)
    for _ in range(2):
        replayed.zero_()
        graph.replay()
        assert torch.equal(c.run(), out)
        torch.cuda.synchronize()
        assert torch.equal(replayed, out)


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_nan_in_launches_of_two_row_blocks(dtype, form):
    users, n, m, at, bad_user, d, heads = 33, 230, 200, 140, 5, 512, 8
    assert attend_rule([m] * users, [n] * users, heads, d // heads)["blocks"] == 2
    c = Case(d, heads, dtype, form, [n] * users, [m] * users, seed=241, check=(bad_user,))
    clean = c.run(causal=True)
    c.check(clean, causal=True, users=(bad_user,))
    for what in "kv":
        k, v = (torch.from_numpy(x[bad_user]).to(TORCH[dtype]).to(DEV).view(n, d) for x in (c.k, c.v))
        (k if what == "k" else v)[at, 64 + 5] = float("nan")
        rg.relaygr_kv_pool_write(c.pool, 1, rg.KvRows([c.handles[bad_user]], [0, n]), k, v)
        got = c.run(causal=True).view(users, m, heads, 64)
        sees = torch.from_numpy(seen_by_rows(n, m, True) > at)
        cols = torch.zeros(heads, 64, dtype=torch.bool)
        if what == "k":
            cols[1] = True
        else:
            cols[1, 5] = True
        assert torch.equal(torch.isnan(got[bad_user]).cpu(), sees[:, None, None] & cols[None])
        want = clean.view(users, m, heads, 64)
        others = [u for u in range(users) if u != bad_user]
        assert torch.equal(got[others], want[others])
        assert torch.equal(got[bad_user][:, [0] + list(range(2, heads))], want[bad_user][:, [0] + list(range(2, heads))])


@pytest.mark.parametrize("form", ["silu", "softmax"])
def test_calls_of_different_sizes_follow_one_another_across_streams(form):
    """One context on two streams in turn: every call has rows, users and cuts of its own, so that partial sums of one that ran beside the other's
    would show; some join themselves and use the context's counters, some have a launch for it."""
    c = Case(256, 4, "bf16", form, [9000, 7000, 5000], [40, 30, 40], seed=251)
    at = offsets(c.rows)
    batches = []
    for users, rows, itself in (((0, 1), (2, 30), False), ((2,), (1,), True), ((0,), (3,), True), ((0,), (40,), False), ((1, 2), (5, 6), True), ((2,), (40,), False)):
        assert joins_itself(rows, [c.lens[u] for u in users], 4, 64) is itself
        q = torch.cat([c.q[at[u]:at[u] + m] for u, m in zip(users, rows)])
        batches.append((rg.KvRows([c.handles[u] for u in users], offsets(rows)), q))
    want = [rg.relaygr_cache_attend(c.ctx, c.pool, 1, *b) for b in batches]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    outs = [[torch.zeros_like(w) for w in want] for _ in range(8)]
    torch.cuda.synchronize()
    for turn, out in enumerate(outs):
        for i, b in enumerate(batches):
            rg.relaygr_cache_attend(c.ctx, c.pool, 1, *b, out=out[i], stream=streams[(turn + i) % 2])
    torch.cuda.synchronize()
    for turn, out in enumerate(outs):
        for i, w in enumerate(want):
            assert torch.equal(out[i], w), (turn, i)
    whole = c.run()          # and each row against the formula
    c.check(whole)


def bare_context(m):
    """A context whose scratch holds the packed weights, the counters and 256 bytes: no partial sum of a row."""
    full = context_for(m, 1, 1)
    size = -(-m.n_layers * 5 * m.d_model ** 2 * 2 // 256) * 256 + 16384 + 256
    scratch = torch.empty(size, dtype=torch.uint8, device=DEV)
    weights = B.WeightsC(full._layers, *(t.data_ptr() for t in full._keep[-3:]), 0.0)
    handle = C.c_void_p()
    lib = rg.load_library()
    assert lib.relaygr_ctx_create(C.byref(full.cfg), C.byref(weights), scratch.data_ptr(), size, C.byref(handle)) == 0, rg.relaygr_last_error()
    if m.attention != "silu":
        assert lib.relaygr_ctx_set_attention(handle, 1) == 0
    return types.SimpleNamespace(handle=handle, scratch=scratch, keep=full)


@pytest.mark.parametrize("form", ["silu", "softmax"])
@pytest.mark.parametrize("d,heads,dtype", [(256, 4, "bf16"), (256, 8, "fp16"), (128, 1, "bf16")])
def test_a_context_without_room_for_partial_sums(d, heads, dtype, form):
    """Two partial sums of a row take 8 d bytes, more than there are: nothing is cut, however long the histories."""
    bare = bare_context(model(d, heads, dtype, form))
    try:
        for lens, rows in (([5000], [1]), ([3000, 100, 9000], [1, 40, 2]), (LONG_ONE, [3] * 20)):
            assert attend_rule(rows, lens, heads, d // heads)["parts"] > 1
            c = Case(d, heads, dtype, form, lens, rows, seed=271)
            cut = c.run()
            c.ctx = bare
            out = c.run()
            c.check(out)
            c.check(cut)
            c.check(c.run(causal=True), causal=True)
    finally:
        torch.cuda.synchronize()
        rg.load_library().relaygr_ctx_destroy(bare.handle)


def test_two_graphs_of_one_step():
    """A step, the write of a token and its attention, captured for two positions: replayed in turn with eager steps of another entry between them."""
    c = Case(256, 4, "bf16", "softmax", [2000, 900], [1, 1], seed=281)
    h0, h1 = c.handles
    rng = np.random.default_rng(7)

    def fresh():
        return values(rng, 1, 256, "bf16")[0].to(DEV)
    k, v, q = fresh(), fresh(), fresh()
    outs, graphs = [torch.zeros_like(q), torch.zeros_like(q)], []

    def step(handle, pos, out=None, stream=None):
        rg.relaygr_kv_pool_write(c.pool, 1, rg.KvRows([handle], [0, 1], first_token=[pos]), k, v, stream=stream)
        return rg.relaygr_cache_attend(c.ctx, c.pool, 1, rg.KvRows([handle], [0, 1], key_len=[pos + 1]), q, causal=True, out=out, stream=stream)
    for i in range(2):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=side):
            step(h0, 1500 + i, outs[i])
    slab = c.pool.slab.clone()
    for turn in range(3):
        vals = [[fresh() for _ in range(3)] for _ in range(2)]
        want = []
        c.pool.slab.copy_(slab)
        for i in range(2):
            for t, new in zip((k, v, q), vals[i]):
                t.copy_(new)
            want.append(step(h0, 1500 + i))
        c.pool.slab.copy_(slab)
        for i in range(2):
            for t, new in zip((k, v, q), vals[i]):
                t.copy_(new)
            graphs[i].replay()
            step(h1, 600 + turn)
            torch.cuda.synchronize()
        for i in range(2):
            assert torch.equal(outs[i], want[i]), (turn, i)
