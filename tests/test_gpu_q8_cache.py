"""Writing K and V into an 8-bit pool and reading them back, bit for bit against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
from q8_util import BLOCK, TORCH, Entry, held, offsets, pool_for, values

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def read(pool, layer, handles, lens, first=None):
    rows = rg.KvRows(handles, offsets(lens), first_token=first)
    k, v = rg.relaygr_kv_pool_read(pool, layer, rows)
    return k.double().cpu().numpy(), v.double().cpu().numpy()


def same(got, want):
    """Equal values, NaN where NaN is wanted."""
    return np.array_equal(got, want.reshape(got.shape), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,heads", [(128, 4), (256, 4), (256, 8), (512, 8), (512, 4), (1024, 8)])
def test_round_trip_of_ragged_histories(dtype, d, heads):
    lens = [1, 63, 64, 65, 0, 200, 128]
    cfg = rg.make_config(3, d, heads, dtype)
    pool, handles = pool_for(cfg, dtype, lens)
    rng = np.random.default_rng(d + heads)
    for layer in (2, 0):
        (k, k64), (v, v64) = values(rng, sum(lens), d, dtype), values(rng, sum(lens), d, dtype)
        rg.relaygr_kv_pool_write(pool, layer, rg.KvRows(handles, offsets(lens)), k.to(DEV), v.to(DEV))
        gk, gv = read(pool, layer, handles, lens)
        at = offsets(lens)
        for u, n in enumerate(lens):
            s = slice(at[u], at[u + 1])
            assert same(gk[s], held(k64[s].reshape(n, heads, d // heads), dtype)), (layer, u)
            assert same(gv[s], held(v64[s].reshape(n, heads, d // heads), dtype)), (layer, u)


@pytest.mark.parametrize("dtype,d,heads", [("bf16", 256, 4), ("fp16", 128, 4), ("bf16", 512, 4)])
def test_tokens_that_join_one_by_one_or_in_chunks(dtype, d, heads):
    """Kept tokens are rounded again where a larger token raises the scale; a write into the middle ends the entry there."""
    rng = np.random.default_rng(7)
    cfg = rg.make_config(2, d, heads, dtype)
    length = 400
    pool, (h,) = pool_for(cfg, dtype, [length])
    want = [Entry(length, heads, d // heads, dtype) for _ in range(2)]
    steps = [(0, 1), (1, 1), (2, 30), (32, 31), (63, 1), (64, 1), (65, 100), (165, 27), (192, 64), (256, 3), (200, 5), (205, 195), (10, 1)]
    for i, (first, n) in enumerate(steps):
        size = 2.0 ** rng.integers(-12, 9)                      # scales that rise and fall by far more than e4m3 spans
        x = [values(rng, n, d, dtype) for _ in range(2)]
        x = [((t.float() * size).to(TORCH[dtype])) for t, _ in x]
        rg.relaygr_kv_pool_write(pool, 1, rg.KvRows([h], [0, n], first_token=[first]), x[0].to(DEV), x[1].to(DEV))
        for e, t in zip(want, x):
            e.write(first, t.double().numpy().reshape(n, heads, d // heads))
        end = -(-(first + n) // BLOCK) * BLOCK
        got = read(pool, 1, [h], [min(end, length)])
        for g, e, what in zip(got, want, "kv"):
            assert same(g, e.x[:min(end, length)]), (i, what)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_odd_values(dtype):
    """Zeros of both signs, the type's smallest and largest values, infinities and NaN, alone and beside ordinary values."""
    heads, dh = 4, 32
    cfg = rg.make_config(1, heads * dh, heads, dtype)
    fi = torch.finfo(TORCH[dtype])
    rng = np.random.default_rng(1)
    blocks = []
    for odd in ([0.0, -0.0], [fi.smallest_normal, -fi.smallest_normal], [fi.max, fi.min, fi.max / 2], [np.inf, -np.inf], [np.nan], [np.nan, np.inf, fi.max],
                [fi.tiny, fi.max], [1.75, 1.76], [float(np.float32(fi.max) * 0.9375), float(np.float32(fi.max) * 0.97)]):
        for scale in (0.0, 1.0, 2.0 ** -10):
            x = rng.standard_normal((BLOCK, heads, dh)) * scale
            x[rng.integers(0, BLOCK, 9), rng.integers(0, heads - 1, 9), rng.integers(0, dh, 9)] = rng.choice(odd, 9)    # the last head has none
            blocks.append(x)
    t = torch.from_numpy(np.concatenate(blocks).astype(np.float32)).to(TORCH[dtype])
    n = t.shape[0]
    pool, (h,) = pool_for(cfg, dtype, [n])
    rg.relaygr_kv_pool_write(pool, 0, rg.KvRows([h], [0, n]), t.to(DEV), t.to(DEV).flip(0))
    k, v = read(pool, 0, [h], [n])
    assert same(k, held(t.double().numpy(), dtype))
    assert same(v, held(t.double().numpy()[::-1], dtype))


def test_every_value_of_the_types_under_one_scale():
    """All finite values up to 1 of either type, in one long history whose blocks share a largest value."""
    for dtype, heads, dh in (("bf16", 2, 64), ("fp16", 4, 32)):
        bits = torch.arange(0x10000, dtype=torch.int32).to(torch.int16).view(TORCH[dtype]).float()
        x = bits[torch.isfinite(bits) & (bits.abs() <= 1.0)]
        per = BLOCK * dh * heads - heads                          # one feature of each head's first token is the largest
        x = torch.cat([x, torch.zeros(-x.numel() % per)]).view(-1, per)
        blk = torch.ones(x.shape[0], BLOCK * heads * dh)
        blk[:, [i for i in range(BLOCK * heads * dh) if not (i < heads * dh and i % dh == 0)]] = x
        t = blk.view(-1, heads * dh).to(TORCH[dtype])
        pool, (h,) = pool_for(rg.make_config(1, heads * dh, heads, dtype), dtype, [t.shape[0]])
        rg.relaygr_kv_pool_write(pool, 0, rg.KvRows([h], [0, t.shape[0]]), t.to(DEV), t.to(DEV))
        k, v = read(pool, 0, [h], [t.shape[0]])
        want = held(t.double().numpy().reshape(-1, heads, dh), dtype)
        assert same(k, want) and same(v, want)


def test_many_users_columns_of_a_wider_array_and_parts_of_entries():
    """More users than one launch takes, rows that are columns of a projection's output, reads from the middle of a block, targets with
    strides of their own; rows and tokens that are not the call's keep what they held."""
    dtype, d, heads, users = "bf16", 256, 4, 150
    rng = np.random.default_rng(3)
    lens = [int(n) for n in rng.integers(1, 150, users)]
    cfg = rg.make_config(2, d, heads, dtype)
    pool, handles = pool_for(cfg, dtype, lens)
    at = offsets(lens)
    fused, f64 = values(rng, sum(lens), 4 * d, dtype)
    fused = fused.to(DEV)
    rg.relaygr_kv_pool_write(pool, 1, rg.KvRows(handles, at), fused[:, 3 * d:].view(-1, heads, d // heads), fused[:, d:2 * d])
    before = pool.slab.clone()
    first = [int(rng.integers(0, n)) for n in lens]
    part = [int(rng.integers(0, n - f + 1)) for n, f in zip(lens, first)]
    po = offsets(part)
    k = torch.full((sum(part), 2 * d), 7.0, dtype=TORCH[dtype], device=DEV)
    v = torch.full((sum(part) + 2, d + 8), 9.0, dtype=TORCH[dtype], device=DEV)
    rg.relaygr_kv_pool_read(pool, 1, rg.KvRows(handles, po, first_token=first), k[:, d:], v[1:-1, :d])
    assert torch.equal(before, pool.slab)
    assert bool((k[:, :d] == 7.0).all()) and bool((v[:, d:] == 9.0).all()) and bool((v[0] == 9.0).all()) and bool((v[-1] == 9.0).all())
    gk, gv = k[:, d:].double().cpu().numpy(), v[1:-1, :d].double().cpu().numpy()
    for u in range(users):
        x = f64[at[u]:at[u + 1]]
        for got, cols in ((gk, slice(3 * d, 4 * d)), (gv, slice(d, 2 * d))):
            want = held(x[:, cols].reshape(lens[u], heads, d // heads), dtype)[first[u]:first[u] + part[u]]
            assert same(got[po[u]:po[u + 1]], want), u


def test_a_write_leaves_other_layers_entries_and_blocks_alone():
    dtype, d, heads = "fp16", 128, 2
    cfg = rg.make_config(3, d, heads, dtype)
    pool, handles = pool_for(cfg, dtype, [300, 300])
    rng = np.random.default_rng(5)
    for layer in range(3):
        k, _ = values(rng, 600, d, dtype)
        rg.relaygr_kv_pool_write(pool, layer, rg.KvRows(handles, [0, 300, 600]), k.to(DEV), k.to(DEV).flip(0))
    before = [read(pool, layer, handles, [300, 300]) for layer in range(3)]
    slab = pool.slab.clone()
    k, k64 = values(rng, 3, d, dtype)
    rg.relaygr_kv_pool_write(pool, 1, rg.KvRows([handles[1]], [0, 3], first_token=[130]), k.to(DEV), k.to(DEV))
    changed = torch.nonzero(slab != pool.slab).view(-1)
    tile = rg.relaygr_kv_pool_bytes_for_q8(cfg, 64, 64)
    codes = 3 * 128 * d
    entry = 5 * tile                                               # the second entry begins behind the first one's five pages
    for byte in (changed - entry).tolist():
        assert byte // tile == 2, "only the third block of the second entry"
        inside = byte % tile
        assert 128 * d <= inside < 2 * 128 * d if inside < codes else codes + heads * 8 <= inside < codes + 2 * heads * 8
    after = [read(pool, layer, handles, [300, 300]) for layer in range(3)]
    for layer in (0, 2):
        assert all(np.array_equal(a, b) for a, b in zip(before[layer], after[layer]))
    for a, b in zip(before[1], after[1]):
        keep = np.r_[0:300, 300:300 + 130, 300 + 192:600]           # (behind the written tokens the block is zero)
        assert np.array_equal(a[keep], b[keep]) and not b[300 + 133:300 + 192].any()


def test_spill_and_reload_keep_every_bit():
    dtype, d, heads = "bf16", 256, 4
    cfg = rg.make_config(2, d, heads, dtype)
    pool, handles = pool_for(cfg, dtype, [300, 129], extra=8)
    rng = np.random.default_rng(9)
    for layer in range(2):
        k, _ = values(rng, 429, d, dtype)
        rg.relaygr_kv_pool_write(pool, layer, rg.KvRows(handles, [0, 300, 429]), k.to(DEV), k.to(DEV).flip(0))
    want = [read(pool, layer, [handles[1]], [129]) for layer in range(2)]
    host = rg.relaygr_kv_pool_spill(pool, handles[1])
    torch.cuda.synchronize()
    assert host.numel() == rg.relaygr_kv_pool_bytes_for_q8(cfg, 129, 64)
    rg.relaygr_kv_pool_free(pool, handles[1])
    other = rg.relaygr_kv_pool_alloc(pool, 77, 64)                  # takes the first of the freed pages
    again = rg.relaygr_kv_pool_reload(pool, 101, 129, host)
    for layer in range(2):
        assert all(np.array_equal(a, b) for a, b in zip(want[layer], read(pool, layer, [again], [129])))
    ex = rg.Expander(pool, 1 << 24)
    rg.relaygr_expander_retire(ex, again)
    torch.cuda.synchronize()
    rg.relaygr_kv_pool_free(pool, other)
    rg.relaygr_expander_trim(ex, 0)
    torch.cuda.synchronize()
    rg.relaygr_expander_trim(ex, 0)
    h, source = rg.relaygr_expander_lookup(ex, 101)
    for layer in range(2):
        assert all(np.array_equal(a, b) for a, b in zip(want[layer], read(pool, layer, [h], [129]))), source
    torch.cuda.synchronize()
    ex.close()


def test_captured_writes_and_reads_replay_on_new_values():
    dtype, d, heads = "bf16", 256, 4
    pool, handles = pool_for(rg.make_config(1, d, heads, dtype), dtype, [200, 70])
    rng = np.random.default_rng(11)
    lens = [200, 70]
    rows = rg.KvRows(handles, offsets(lens))
    k = torch.zeros(270, d, dtype=TORCH[dtype], device=DEV)
    v, ko, vo = torch.zeros_like(k), torch.empty_like(k), torch.empty_like(k)
    rg.relaygr_kv_pool_write(pool, 0, rows, k, v)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        rg.relaygr_kv_pool_write(pool, 0, rows, k, v)
        rg.relaygr_kv_pool_read(pool, 0, rows, ko, vo)
    for _ in range(3):
        (nk, k64), (nv, v64) = values(rng, 270, d, dtype), values(rng, 270, d, dtype)
        k.copy_(nk.to(DEV))
        v.copy_(nv.to(DEV))
        graph.replay()
        torch.cuda.synchronize()
        for got, x in ((ko, k64), (vo, v64)):
            want = np.concatenate([held(x[:200].reshape(200, heads, d // heads), dtype), held(x[200:].reshape(70, heads, d // heads), dtype)])
            assert same(got.double().cpu().numpy(), want)
        eager = rg.relaygr_kv_pool_read(pool, 0, rows)
        assert torch.equal(eager[0], ko) and torch.equal(eager[1], vo)


def test_calls_on_a_side_stream_and_results_made_there():
    dtype, d, heads = "fp16", 256, 8
    pool, (h,) = pool_for(rg.make_config(1, d, heads, dtype), dtype, [1000])
    rng = np.random.default_rng(13)
    (k, k64), (v, v64) = values(rng, 1000, d, dtype), values(rng, 1000, d, dtype)
    k, v = k.to(DEV), v.to(DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    rows = rg.KvRows([h], [0, 1000])
    for stream in (side, int(side.cuda_stream)):
        rg.relaygr_kv_pool_write(pool, 0, rows, k, v, stream=stream)
        gk, gv = rg.relaygr_kv_pool_read(pool, 0, rows, stream=stream)
        side.synchronize()
        assert same(gk.double().cpu().numpy(), held(k64.reshape(1000, heads, d // heads), dtype))
        assert same(gv.double().cpu().numpy(), held(v64.reshape(1000, heads, d // heads), dtype))


@pytest.mark.parametrize("dtype,d,heads", [("bf16", 256, 4), ("fp16", 256, 8), ("bf16", 1024, 8)])
def test_batches_that_the_caches_do_not_hold(dtype, d, heads):
    """128 MiB of rows and codes and more move by kernels that leave nothing in the caches: all of it written, its second part from the middle of a
    block again, and read; three of the users against the definition."""
    rng = np.random.default_rng(41)
    users = 28
    lens = [int(n) for n in rng.integers(3900, 4100, users) * 256 // d]
    kept = [n - int(rng.integers(64, 200)) for n in lens]
    cfg = rg.make_config(1, d, heads, dtype)
    pool, handles = pool_for(cfg, dtype, lens)
    at, pick = offsets(lens), (0, 11, users - 1)
    assert sum(lens) * d * 6 >= 128 << 20
    x = [torch.randn(sum(lens), d, device=DEV).to(TORCH[dtype]) for _ in range(2)]
    rg.relaygr_kv_pool_write(pool, 0, rg.KvRows(handles, at), *x)
    got = rg.relaygr_kv_pool_read(pool, 0, rg.KvRows(handles, at))
    for g, t in zip(got, x):
        for u in pick:
            want = held(t[at[u]:at[u + 1]].double().cpu().numpy().reshape(lens[u], heads, d // heads), dtype)
            assert same(g[at[u]:at[u + 1]].double().cpu().numpy(), want), u
    # the users' last tokens eight times as large (launched with the others' unchanged ones, so that the batch is as large as before)
    first = [k if u in pick else 0 for u, k in enumerate(kept)]
    rows = offsets([n - f for n, f in zip(lens, first)])
    part = [torch.cat([t[at[u] + first[u]:at[u + 1]] * (8.0 if u in pick else 1.0) for u in range(users)]) for t in x]
    assert int(rows[-1]) * d * 6 >= 128 << 20
    rg.relaygr_kv_pool_write(pool, 0, rg.KvRows(handles, rows, first_token=first), *part)
    again = rg.relaygr_kv_pool_read(pool, 0, rg.KvRows(handles, at))
    for g, before, t in zip(again, got, x):
        for u in range(users):
            a = slice(int(at[u]), int(at[u + 1]))
            if u not in pick:
                assert torch.equal(g[a], before[a]), u
                continue
            e = Entry(lens[u], heads, d // heads, dtype)
            y = t[a].double().cpu().numpy().reshape(lens[u], heads, d // heads)
            e.write(0, y)
            e.write(first[u], 8.0 * y[first[u]:])
            assert same(g[a].double().cpu().numpy(), e.x), u
