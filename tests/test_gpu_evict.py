"""Eviction from an 8-bit pool against its definition: which tokens stay, and what the cache then stands for."""
import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
from q8_util import TORCH, context_for, held, model, offsets, pool_for, values
from scored_util import scored, visible

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def choose(w, keep, first, recent):
    """Places that stay: those that must, then the largest weights, ties to the lowest place; NaN below all."""
    n = len(w)
    if keep == n:
        return np.arange(n)
    order = sorted(range(first, n - recent), key=lambda j: (1, 0.0, j) if np.isnan(w[j]) else (0, -float(w[j]), j))
    return np.sort(np.concatenate([np.arange(first), np.asarray(order[:keep - first - recent], np.int64), np.arange(n - recent, n)]).astype(np.int64))


class Case:
    """Entries of the given lengths with values in every layer, held in 64 bits too, and weights and positions with gaps between users."""

    def __init__(self, d, heads, dtype, lens, seed=0, layers=2, spread=0.6, page_tokens=64, wild=False, to_lens=None):
        self.d, self.heads, self.dtype, self.lens, self.layers = d, heads, dtype, lens, layers
        self.rng = np.random.default_rng(seed)
        self.cfg = rg.make_config(layers, d, heads, dtype)
        self.pool, handles = pool_for(self.cfg, dtype, list(lens) + list(to_lens or []), page_tokens)
        self.handles, self.to = handles[:len(lens)], handles[len(lens):]
        at = offsets(lens)
        self.kv = []
        for layer in range(layers):
            pair = []
            for _ in range(2):
                x, _ = values(self.rng, sum(lens), d, dtype, spread)
                if wild:      # blocks whose tokens differ by powers of two: scales that differ, codes that become subnormal
                    x = (x.float() * torch.from_numpy(np.exp2(self.rng.integers(-14, 8, (sum(lens), 1))).astype(np.float32))).to(TORCH[dtype])
                pair.append(x)
            rg.relaygr_kv_pool_write(self.pool, layer, rg.KvRows(self.handles, at), pair[0].to(DEV), pair[1].to(DEV))
            self.kv.append([[held(x.double().numpy()[at[u]:at[u + 1]].reshape(n, heads, d // heads), dtype) for u, n in enumerate(lens)] for x in pair])
        self.token_off = np.cumsum([2] + [n + 3 for n in lens])[:-1]
        self.n_tokens = int(self.token_off[-1] + lens[-1] + 4)
        self.w = np.exp(2 * self.rng.standard_normal(self.n_tokens)).astype(np.float32)
        self.w[self.rng.random(self.n_tokens) < 0.2] = 0.0
        self.pos = self.rng.integers(0, 1 << 20, self.n_tokens).astype(np.int32)

    def mine(self, x, u):
        return x[self.token_off[u]:self.token_off[u] + self.lens[u]]

    def evict(self, keep, first=0, recent=0, to=None, **kw):
        rows = rg.KvRows(self.handles, offsets(keep), key_len=self.lens)
        self.weight_out, self.pos_out = torch.full((sum(keep) + 1,), -7.0, device=DEV), torch.full((sum(keep) + 1,), -7, dtype=torch.int32, device=DEV)
        return rg.relaygr_kv_pool_evict(self.pool, rows, torch.from_numpy(self.w).to(DEV), self.token_off, first, recent, to=to, weight_out=self.weight_out,
                                        position=torch.from_numpy(self.pos).to(DEV), position_out=self.pos_out, **kw)

    def check(self, kept, keep, first=0, recent=0, to=None):
        ko = offsets(keep)
        kept = kept.cpu().numpy()
        w, pos = self.weight_out.cpu().numpy(), self.pos_out.cpu().numpy()
        assert w[-1] == -7.0 and pos[-1] == -7
        handles = self.handles if to is None else to
        for u, m in enumerate(keep):
            want = choose(self.mine(self.w, u), m, first, recent) if m else np.zeros(0, np.int64)
            got = kept[ko[u]:ko[u + 1]]
            assert np.array_equal(got, want), (u, m)
            assert np.array_equal(w[ko[u]:ko[u + 1]], self.mine(self.w, u)[want], equal_nan=True) and np.array_equal(pos[ko[u]:ko[u + 1]], self.mine(self.pos, u)[want])
            if m == 0:
                continue
            whole = min(-(-m // 64) * 64, rg.relaygr_kv_pool_entry_len(self.pool, int(handles[u])))
            for layer in range(self.layers):
                for x, read in zip(self.kv[layer], rg.relaygr_kv_pool_read(self.pool, layer, rg.KvRows([handles[u]], [0, whole]))):
                    read = read.double().cpu().numpy()
                    assert np.array_equal(read[:m], held(x[u][want], self.dtype).reshape(m, self.d), equal_nan=True), (u, layer)
                    assert (read[m:] == 0).all(), "behind the last token"


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,heads", [(128, 4), (256, 4), (512, 8), (1024, 8), (128, 1)])
def test_ragged_histories_in_place_and_elsewhere(d, heads, dtype):
    lens = [1, 64, 65, 200, 63, 700, 129, 1500]
    keep = [1, 30, 64, 65, 63, 257, 0, 1000]
    for seed, (first, recent) in enumerate(((0, 0), (4, 20), (1, 0), (0, 29))):
        c = Case(d, heads, dtype, lens, seed=d + seed, to_lens=[max(m, 1) for m in keep])
        kept = c.evict(keep, first, recent, to=c.to)
        c.check(kept, keep, first, recent, to=c.to)
        # the entries it came from are as they were
        k, v = rg.relaygr_kv_pool_read(c.pool, 1, rg.KvRows(c.handles, offsets(lens)))
        assert np.array_equal(k.double().cpu().numpy(), np.concatenate([x.reshape(-1, d) for x in c.kv[1][0]]))
        c.check(c.evict(keep, first, recent), keep, first, recent)
        # an entry of which nothing stays is left alone
        k, _ = rg.relaygr_kv_pool_read(c.pool, 0, rg.KvRows([c.handles[6]], [0, 129]))
        assert np.array_equal(k.double().cpu().numpy(), c.kv[0][0][6].reshape(129, d))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_blocks_whose_scales_differ(dtype):
    lens, keep = [900, 640, 100], [300, 500, 64]
    c = Case(256, 4, dtype, lens, seed=5, wild=True)
    c.check(c.evict(keep, 3, 10), keep, 3, 10)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 1023, 1024, 1025, 5000])
def test_counts_ties_and_odd_weights(n):
    """Every count of a short history; equal weights, zeros of both signs, infinities, NaN and subnormal weights."""
    c = Case(128, 4, "bf16", [n], seed=n, layers=1)
    rng = np.random.default_rng(n)
    specials = np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 1e-42, -1e-42, 1.0, -1.0, 3.4e38], np.float32)
    for kind in range(3):
        if kind == 0:
            w = rng.choice(specials, n)
        elif kind == 1:
            w = np.full(n, 0.25, np.float32)
        else:
            w = np.float32(1.0) + np.arange(n, dtype=np.float32) % 7 * np.float32(2.0 ** -23)
        c.w[c.token_off[0]:c.token_off[0] + n] = w
        for m in sorted({1, 2, n // 2, n - 1, n} - {0}):
            if m > n:
                continue
            for first, recent in ((0, 0), (1, 0), (0, 1), (min(2, m) // 2, m // 3)):
                if first + recent > m:
                    continue
                rows = rg.KvRows(c.handles, [0, m], key_len=[n])
                scratch = rg.relaygr_kv_pool_alloc(c.pool, 99, min(n, 128)) if m <= 128 else None
                if scratch is None:
                    continue
                kept = rg.relaygr_kv_pool_evict(c.pool, rows, torch.from_numpy(c.w).to(DEV), c.token_off, first, recent, to=[scratch])
                assert np.array_equal(kept.cpu().numpy(), choose(w, m, first, recent)), (kind, m, first, recent)
                rg.relaygr_kv_pool_free(c.pool, scratch)
    m = n - n // 3
    c.w[c.token_off[0]:c.token_off[0] + n] = rng.choice(specials, n)
    kept = c.evict([m], 0, n // 4)
    c.check(kept, [m], 0, n // 4)


@pytest.mark.parametrize("kind", ["specials", "equal", "a step apart"])
@pytest.mark.parametrize("n", [255, 256, 257, 1023, 1024, 1025, 2047, 2048, 2049, 4095, 4096, 4097, 5000, 33000])
def test_large_counts_of_ties_and_odd_weights(n, kind):
    """Counts around the choosing's spans of tokens (1024 threads of four; 4096 tokens in registers, 32 768 in LDS), where ties lie in several of them."""
    c = Case(128, 4, "bf16", [n], seed=n, layers=1, to_lens=[n])
    rng = np.random.default_rng(n)
    if kind == "specials":
        w = rng.choice(np.array([0.0, -0.0, np.inf, -np.inf, np.nan, 1e-42, -1e-42, 1.0, -1.0, 3.4e38], np.float32), n)
    elif kind == "equal":
        w = np.full(n, 0.25, np.float32)
    else:
        w = np.float32(1.0) + np.arange(n, dtype=np.float32) % 7 * np.float32(2.0 ** -23)
    c.w[c.token_off[0]:c.token_off[0] + n] = w
    for m in sorted({m for m in (129, n // 2, n // 2 + 1, 1024, 1025, 4096, n - 1, n) if m <= n}):
        for first, recent in ((0, 0), (1, 0), (0, 1), (1, m // 3), (m // 2, m - m // 2), (m // 2, m - m // 2 - 1)):
            kept = c.evict([m], first, recent, to=c.to)
            want = choose(w, m, first, recent)
            assert np.array_equal(kept.cpu().numpy(), want), (m, first, recent)
            assert np.array_equal(c.weight_out.cpu().numpy()[:m], w[want], equal_nan=True) and np.array_equal(c.pos_out.cpu().numpy()[:m], c.mine(c.pos, 0)[want])
    c.check(c.evict([m - 1], 0, n // 4, to=c.to), [m - 1], 0, n // 4, to=c.to)
    c.check(c.evict([m - 1], 0, n // 4), [m - 1], 0, n // 4)


@pytest.mark.parametrize("n", [4095, 4096, 4097, 16385, 32768, 32769, 40001])
def test_long_entries(n):
    """Lengths around what the choosing holds in registers and in LDS: weights of many values and of few, whose ties lie in several spans of tokens; weights and positions over themselves."""
    c = Case(128, 2, "fp16", [n], seed=n, layers=1, to_lens=[n])
    rng = np.random.default_rng(n)
    for few in (False, True):
        mine = slice(c.token_off[0], c.token_off[0] + n)
        c.w[mine] = rng.integers(0, 3, n) if few else np.exp(2 * rng.standard_normal(n))
        for m, first, recent in ((n - 1, 4, 100), (n // 2, 0, 0), (n // 3, 5000 if n > 16384 else 1, 64)):
            rows = rg.KvRows(c.handles, [0, m], key_len=[n])
            weight, position = torch.from_numpy(c.w.copy()).to(DEV), torch.from_numpy(c.pos).to(DEV)
            other = int(c.to[0])
            kept = rg.relaygr_kv_pool_evict(c.pool, rows, weight, c.token_off, first, recent, to=[other], weight_out=weight, position=position, position_out=position,
                                            out_off=c.token_off).cpu().numpy()
            want = choose(c.w[mine], m, first, recent)
            assert np.array_equal(kept, want), (few, m)
            at = np.arange(n)[:m] + c.token_off[0]
            expected_w, expected_pos = c.w.copy(), c.pos.copy()
            expected_w[at], expected_pos[at] = c.w[mine][want], c.pos[mine][want]
            assert np.array_equal(weight.cpu().numpy(), expected_w) and np.array_equal(position.cpu().numpy(), expected_pos)
            for x, read in zip(c.kv[0], rg.relaygr_kv_pool_read(c.pool, 0, rg.KvRows([other], [0, m]))):
                assert np.array_equal(read.double().cpu().numpy(), held(x[0][want], "fp16").reshape(m, 128))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,heads", [(256, 8), (512, 8), (1024, 8)])
def test_in_place_by_few_and_by_many_workgroups(d, heads, dtype):
    """Histories of many tiles, a few of them and so many that the launch takes narrower workgroups."""
    for lens in ([5000, 1030], [int(n) for n in np.random.default_rng(d).integers(300, 700, 18)]):
        for of in (0.3, 0.97):
            keep = [int(of * n) for n in lens]
            c = Case(d, heads, dtype, lens, seed=d, layers=2)
            c.check(c.evict(keep, 2, 50), keep, 2, 50)


def test_many_users_and_what_lies_beside_them():
    """More users than a launch takes; other entries, and blocks behind what stays, keep every bit."""
    lens = [int(x) for x in np.random.default_rng(3).integers(1, 400, 150)]
    keep = [n if u % 7 == 0 else max(1, n // 2) for u, n in enumerate(lens)]
    for to in (False, True):
        c = Case(128, 2, "fp16", lens, seed=4, layers=1, to_lens=keep if to else None)
        spare = rg.relaygr_kv_pool_alloc(c.pool, 7777, 128)
        before = c.pool.slab.clone()
        kept = c.evict(keep, 0, 1, to=c.to if to else None)
        c.check(kept, keep, 0, 1, to=c.to if to else None)
        tile = rg.relaygr_kv_pool_bytes_for_q8(c.cfg, 64, 64)
        written = np.zeros(c.pool.slab.numel(), bool)
        for h, m in zip(c.to if to else c.handles, keep):
            at = rg.relaygr_kv_pool_locate(c.pool, h, 0, 0, 0)[0]
            written[at:at + -(-m // 64) * tile] = True
        same = (c.pool.slab == before).cpu().numpy()
        assert same[~written].all()
        assert rg.relaygr_kv_pool_entry_len(c.pool, spare) == 128


def test_nan_codes_and_the_types_largest_values_stay():
    for dtype in ("bf16", "fp16"):
        c = Case(128, 2, dtype, [200], seed=6, layers=1)
        top = torch.finfo(TORCH[dtype]).max
        k = torch.randn((200, 128), device=DEV).to(TORCH[dtype])
        k[10, 3], k[70, 100], k[150, 5], k[199, 64] = float("nan"), top, -top, float("inf")
        rg.relaygr_kv_pool_write(c.pool, 0, rg.KvRows(c.handles, [0, 200]), k, k)
        c.kv[0] = [[held(k.double().cpu().numpy().reshape(200, 2, 64), dtype)] for _ in range(2)]
        c.w[:] = 1.0
        c.w[c.token_off[0] + np.arange(20, 60)] = 0.0
        c.check(c.evict([160]), [160])


def test_in_place_arrays_and_repeated_eviction():
    """A history that is cut again and again: weights and positions shrink where they stand."""
    d, heads, dtype, n = 256, 4, "bf16", 3000
    c = Case(d, heads, dtype, [n, 500], seed=8)
    w, pos = torch.from_numpy(c.w).to(DEV), torch.from_numpy(c.pos).to(DEV)
    lens = [n, 500]
    for keep in ([2000, 500], [1999, 131], [640, 1]):
        rows = rg.KvRows(c.handles, offsets(keep), key_len=lens)
        before_w, before_p = w.cpu().numpy(), pos.cpu().numpy()
        kept = rg.relaygr_kv_pool_evict(c.pool, rows, w, c.token_off, first=1, weight_out=w, position=pos, position_out=pos, out_off=c.token_off).cpu().numpy()
        after_w, after_p = w.cpu().numpy(), pos.cpu().numpy()
        for u, (m, o) in enumerate(zip(keep, c.token_off)):
            want = choose(before_w[o:o + lens[u]], m, 1 if m < lens[u] else 0, 0)
            assert np.array_equal(kept[offsets(keep)[u]:offsets(keep)[u + 1]], want)
            assert np.array_equal(after_w[o:o + m], before_w[o:o + lens[u]][want]) and np.array_equal(after_p[o:o + m], before_p[o:o + lens[u]][want])
            assert np.array_equal(after_w[o + m:o + lens[u] + 3], before_w[o + m:o + lens[u] + 3])
            for layer in range(2):
                for x in c.kv[layer]:
                    x[u] = held(x[u][want], dtype)
                k, v = rg.relaygr_kv_pool_read(c.pool, layer, rg.KvRows([c.handles[u]], [0, m]))
                assert np.array_equal(k.double().cpu().numpy(), c.kv[layer][0][u].reshape(m, d)) and np.array_equal(v.double().cpu().numpy(), c.kv[layer][1][u].reshape(m, d))
        lens = keep


def test_captured_eviction_replays_on_new_weights():
    c = Case(256, 4, "bf16", [700, 300], seed=12, to_lens=[400, 100])
    rows = rg.KvRows(c.handles, [0, 400, 500], key_len=c.lens)
    w = torch.from_numpy(c.w).to(DEV)
    kept = torch.empty(500, dtype=torch.int32, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rg.relaygr_kv_pool_evict(c.pool, rows, w, c.token_off, 2, 3, to=c.to, kept=kept)
    for turn in range(3):
        c.w = np.random.default_rng(turn).random(c.n_tokens).astype(np.float32)
        w.copy_(torch.from_numpy(c.w))
        graph.replay()
        torch.cuda.synchronize()
        for u, (m, o) in enumerate(((400, 0), (100, 400))):
            want = choose(c.mine(c.w, u), m, 2, 3)
            assert np.array_equal(kept[o:o + m].cpu().numpy(), want)
            k, _ = rg.relaygr_kv_pool_read(c.pool, 1, rg.KvRows([c.to[u]], [0, m]))
            assert np.array_equal(k.double().cpu().numpy(), held(c.kv[1][0][u][want], "bf16").reshape(m, 256))


def test_entries_beyond_4_gib_of_the_slab():
    d, heads, dtype = 1024, 8, "bf16"
    cfg = rg.make_config(16, d, heads, dtype)
    tile = rg.relaygr_kv_pool_bytes_for_q8(cfg, 64, 64)
    before = (1 << 32) // tile + 3
    pool = rg.KvPool(cfg, dtype, (before + 6) * tile, 64, quantized=True)
    pool.slab.fill_(0x7F)
    rg.relaygr_kv_pool_alloc(pool, 1, before * 64)
    h = rg.relaygr_kv_pool_alloc(pool, 2, 300)
    rng = np.random.default_rng(67)
    k, k64 = values(rng, 300, d, dtype)
    for layer in range(16):
        rg.relaygr_kv_pool_write(pool, layer, rg.KvRows([h], [0, 300]), k.to(DEV), k.to(DEV))
    w = rng.random(300).astype(np.float32)
    kept = rg.relaygr_kv_pool_evict(pool, rg.KvRows([h], [0, 130]), torch.from_numpy(w).to(DEV), [0])
    want = choose(w, 130, 0, 0)
    assert np.array_equal(kept.cpu().numpy(), want)
    values_kept = held(held(k64.reshape(300, heads, -1), dtype)[want], dtype).reshape(130, d)
    for layer in (0, 15):
        for got in rg.relaygr_kv_pool_read(pool, layer, rg.KvRows([h], [0, 130])):
            assert np.array_equal(got.double().cpu().numpy(), values_kept)


def test_a_history_that_goes_on_growing():
    """Rows are turned by their positions, written, attend with a bias by distance and add up the tokens' weights; a full entry is cut back to its recent and its heaviest
    tokens, and the history goes on.  Every step against the same in 64 bits on what the cache holds."""
    d, heads, dtype, room = 256, 4, "bf16", 192
    dh = d // heads
    rng = np.random.default_rng(21)
    ctx = context_for(model(d, heads, dtype, "softmax"), 2, 64)
    cfg = ctx.cfg
    pool, handles = pool_for(cfg, dtype, [room, room])
    rope = rg.Rope(dh)
    slopes = torch.tensor([0.5, 0.1, 0.02, 0.004], device=DEV)
    token_off = [0, room]
    weight, position = torch.zeros(2 * room, device=DEV), torch.zeros(2 * room, dtype=torch.int32, device=DEV)
    lens, seen = [0, 0], [0, 0]
    total, dtotal = [np.zeros(0), np.zeros(0)], [np.zeros(0), np.zeros(0)]
    evictions = 0
    for step in range(14):
        new = [int(rng.integers(1, 40)), 17]
        if any(n + m > room for n, m in zip(lens, new)):
            keep = [min(n, 100) for n in lens]
            rows = rg.KvRows(handles, offsets(keep), key_len=lens)
            before = weight.double().cpu().numpy()
            kept = rg.relaygr_kv_pool_evict(pool, rows, weight, token_off, 4, 30, weight_out=weight, position=position, position_out=position, out_off=token_off).cpu().numpy()
            at = offsets(keep)
            for u in range(2):
                mine = kept[at[u]:at[u + 1]]
                assert np.array_equal(mine, choose(before[token_off[u]:token_off[u] + lens[u]], keep[u], 4 if keep[u] < lens[u] else 0, 30 if keep[u] < lens[u] else 0))
                total[u], dtotal[u] = total[u][mine], dtotal[u][mine]
            weight[keep[0]:room] = 0.0
            weight[room + keep[1]:] = 0.0
            lens = keep
            evictions += 1
        at = offsets(new)
        row_pos = np.concatenate([s + np.arange(m) for s, m in zip(seen, new)]).astype(np.int32)
        pos = torch.from_numpy(row_pos).to(DEV)
        q, k, v = (values(rng, sum(new), d, dtype)[0].to(DEV) for _ in range(3))
        q, k = rg.relaygr_rotary(cfg, rope, pos, q, k)
        rg.relaygr_kv_pool_write(pool, 1, rg.KvRows(handles, at, first_token=lens), k, v)
        for u in range(2):
            position[token_off[u] + lens[u]:token_off[u] + lens[u] + new[u]] = pos[at[u]:at[u + 1]]
        lens, seen = [n + m for n, m in zip(lens, new)], [s + m for s, m in zip(seen, new)]
        scoring = rg.Scoring(cap=20.0, slopes=slopes, row_position=pos, key_position=position, token_off=token_off)
        out = rg.relaygr_cache_attend_scored(ctx, pool, 1, rg.KvRows(handles, at, key_len=lens), q, scoring, causal=True, weight=weight).double().cpu().numpy()
        for u in range(2):
            kh, vh = (x.double().cpu().numpy().reshape(lens[u], heads, dh) for x in rg.relaygr_kv_pool_read(pool, 1, rg.KvRows([handles[u]], [0, lens[u]])))
            key_pos = position[token_off[u]:token_off[u] + lens[u]].cpu().numpy()
            want, bound, t, dt = scored(q.double().cpu().numpy()[at[u]:at[u + 1]].reshape(new[u], heads, dh), kh, vh, visible(lens[u], new[u], True), "softmax", dtype, 20.0,
                                        slopes.cpu().numpy(), row_pos[at[u]:at[u + 1]], key_pos)
            assert (np.abs(out[at[u]:at[u + 1]].reshape(want.shape) - want) <= bound).all(), (step, u)
            total[u] = np.concatenate([total[u], np.zeros(new[u])]) + t
            dtotal[u] = np.concatenate([dtotal[u], np.zeros(new[u])]) + dt + 2.0 ** -23 * total[u]
            got = weight[token_off[u]:token_off[u] + lens[u]].double().cpu().numpy()
            assert (np.abs(got - total[u]) <= dtotal[u]).all(), (step, u)
    assert evictions >= 2


def test_refusals():
    c = Case(256, 4, "bf16", [100, 50], seed=59, to_lens=[64, 50])
    w, p = torch.zeros(c.n_tokens, device=DEV), torch.zeros(c.n_tokens, dtype=torch.int32, device=DEV)
    before = c.pool.slab.clone()

    def code(handles=None, keep=(60, 40), key_len=(100, 50), weight=w, token_off=c.token_off, pool=None, **kw):
        rows = rg.KvRows(c.handles if handles is None else handles, offsets(keep), key_len=key_len)
        with pytest.raises(rg.RelayGRError) as e:
            rg.relaygr_kv_pool_evict(pool or c.pool, rows, weight, token_off, **kw)
        torch.cuda.synchronize()
        assert torch.equal(c.pool.slab, before)
        return e.value.code
    a, b = c.handles
    for kw in (dict(key_len=(101, 50)), dict(keep=(60, 51)), dict(key_len=(-1, 50), keep=(0, 1)), dict(first=-1), dict(recent=-1), dict(first=20, recent=21), dict(to=[c.to[0], a]), dict(to=[c.to[1], c.to[1]]),
               dict(keep=(65, 40), to=c.to), dict(handles=[a, a]), dict(token_off=[0]), dict(token_off=[-5, 10]), dict(token_off=[c.n_tokens - 99, 0]), dict(weight=w.half()), dict(weight=w.cpu()),
               dict(kept=torch.zeros(99, dtype=torch.int32, device=DEV)), dict(kept=torch.zeros(100, device=DEV)), dict(weight_out=w[:99]), dict(position_out=p), dict(position=p[:50], position_out=p),
               dict(weight_out=w), dict(weight_out=w, out_off=[c.token_off[0] + 1, c.token_off[1]]), dict(weight_out=w.clone(), out_off=[0, 59]), dict(out_off=[-1, 60], weight_out=w.clone()),
               dict(weight_out=w.double()), dict(to=[a])):
        assert code(**kw) == rg.RELAYGR_EINVAL, kw
    assert code(handles=[a, 12345]) == rg.RELAYGR_ENOENT and code(to=[c.to[0], 12345]) == rg.RELAYGR_ENOENT
    p16 = rg.KvPool(c.cfg, "bf16", 4 * rg.relaygr_kv_pool_bytes_for(c.cfg, 64, 64), 64)
    h16 = rg.relaygr_kv_pool_alloc(p16, 1, 100)
    assert code(pool=p16, handles=[h16], keep=(10,), key_len=(100,), token_off=[0]) == rg.RELAYGR_EINVAL
    assert rg.relaygr_kv_pool_evict(c.pool, rg.KvRows([], [0]), w[:0], []).numel() == 0
    assert rg.relaygr_kv_pool_evict(c.pool, rg.KvRows([a, a], [0, 0, 0]), w, [0, 0]).numel() == 0
