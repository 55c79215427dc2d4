"""The 8-bit pool and its calls without a GPU: sizes, the allocator, where codes are, and every refusal that the host makes before anything
is enqueued.  The slab's address is never dereferenced."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
from paper_2601_01712_amd import binding as B
from q8_util import attend_rule, e4m3, exponent, held, rule_shim

CFG = dict(n_layers=3, d_model=256, n_heads=4, dtype="bf16")


class FakePool:
    """An 8-bit (or 16-bit) pool over addresses nobody reads."""

    def __init__(self, cfg, pages=10, page_tokens=128, q8=True):
        lib = rg.load_library()
        self.cfg, self.dtype = cfg, "bf16"
        size = (rg.relaygr_kv_pool_bytes_for_q8 if q8 else rg.relaygr_kv_pool_bytes_for)(cfg, page_tokens, page_tokens)
        self.handle = C.c_void_p()
        create = lib.relaygr_kv_pool_create_q8 if q8 else lib.relaygr_kv_pool_create
        assert create(C.byref(cfg), C.c_void_p(0x10000000), pages * size, page_tokens, C.byref(self.handle)) == 0, rg.relaygr_last_error()

    def __del__(self):
        rg.load_library().relaygr_kv_pool_destroy(self.handle)


def test_sizes():
    cfg = rg.make_config(8, 512, 8, "bf16")
    codes, scales = 2 * 8 * 512, 2 * 8 * 8 * 4
    assert rg.relaygr_kv_footprint_bytes_q8(cfg, 8192) == 8192 * codes + 128 * scales
    assert rg.relaygr_kv_footprint_bytes_q8(cfg, 65) == 65 * codes + 2 * scales
    assert rg.relaygr_kv_pool_bytes_for_q8(cfg, 8192, 256) == 128 * (64 * codes + scales)
    assert rg.relaygr_kv_pool_bytes_for_q8(cfg, 8193, 256) == 132 * (64 * codes + scales)
    assert rg.relaygr_kv_pool_bytes_for_q8(cfg, 0, 256) == 0
    assert rg.relaygr_kv_pool_bytes_for_q8(cfg, 8192, 256) < 0.51 * rg.relaygr_kv_pool_bytes_for(cfg, 8192, 256)
    # scales are padded to whole 128-byte lines
    small = rg.make_config(1, 128, 2, "fp16")
    assert rg.relaygr_kv_pool_bytes_for_q8(small, 64, 64) == 64 * 2 * 128 + 128
    for bad in (rg.make_config(2, 256, 4, "fp32"), rg.make_config(0, 256, 4, "bf16")):
        assert rg.relaygr_kv_footprint_bytes_q8(bad, 100) == 0 and rg.relaygr_kv_pool_bytes_for_q8(bad, 100, 64) == 0
    assert rg.relaygr_kv_pool_bytes_for_q8(cfg, 100, 65) == 0 and rg.relaygr_kv_footprint_bytes_q8(cfg, -1) == 0


def test_creation_refuses_fp32_and_bad_slabs():
    lib, out = rg.load_library(), C.c_void_p()

    def create(cfg, slab, n, page):
        return lib.relaygr_kv_pool_create_q8(C.byref(cfg), C.c_void_p(slab), n, page, C.byref(out))
    cfg = rg.make_config(**CFG)
    assert create(rg.make_config(2, 256, 4, "fp32"), 0x10000000, 1 << 24, 64) == rg.RELAYGR_EINVAL
    assert create(cfg, 0x10000010, 1 << 24, 64) == rg.RELAYGR_EINVAL
    assert create(cfg, 0x10000000, 1 << 24, 100) == rg.RELAYGR_EINVAL
    assert create(cfg, 0x10000000, 1 << 10, 64) == rg.RELAYGR_ENOSPC
    assert out.value is None


def test_allocator_and_where_codes_are():
    cfg = rg.make_config(**CFG)
    p = FakePool(cfg)
    a, b = rg.relaygr_kv_pool_alloc(p, 1, 100), rg.relaygr_kv_pool_alloc(p, 2, 300)
    assert rg.relaygr_kv_pool_stats(p) == {"pages_total": 10, "pages_free": 6, "live_entries": 2, "largest_free_extent": 6}
    assert rg.relaygr_kv_pool_entry_bytes(p, b) == rg.relaygr_kv_pool_bytes_for_q8(cfg, 300, 128)
    # every byte of the codes of an entry belongs to one element, and codes lie before the tile's scales
    tile = rg.relaygr_kv_pool_bytes_for_q8(cfg, 64, 64)
    assert tile == 3 * 128 * 256 + 128        # (3 layers x 4 heads x 2 scales: 96 bytes, padded)
    seen = set()
    for token in (0, 1, 37, 63, 64, 99):
        for layer in range(3):
            for f in range(0, 256, 5):
                k, v = rg.relaygr_kv_pool_locate(p, a, layer, token, f)
                assert k // tile == v // tile == token // 64 and k % tile < 3 * 128 * 256 and v % tile < 3 * 128 * 256
                assert (k % tile) // (128 * 256) == layer == (v % tile) // (128 * 256)
                seen |= {k, v}
    assert len(seen) == 2 * 6 * 3 * 52
    assert rg.relaygr_kv_pool_locate(p, b, 0, 0, 0)[0] == 2 * tile      # a page is 128 tokens
    rg.relaygr_kv_pool_free(p, a)
    with pytest.raises(rg.RelayGRError) as e:
        rg.relaygr_kv_pool_locate(p, a, 0, 0, 0)
    assert e.value.code == rg.RELAYGR_ENOENT


def _call(p, name, layer, rows, k=0x1000, ks=256, v=0x2000, vs=256):
    lib = rg.load_library()
    rc = getattr(lib, name)(p.handle, layer, C.byref(rows.c) if rows is not None else None, k, ks, v, vs, None)
    return rc, rg.relaygr_last_error()


@pytest.mark.parametrize("name", ["relaygr_kv_pool_write", "relaygr_kv_pool_read"])
def test_write_and_read_refuse(name):
    cfg = rg.make_config(**CFG)
    p = FakePool(cfg)
    h = [rg.relaygr_kv_pool_alloc(p, u, 100) for u in range(3)]
    ok = rg.KvRows(h, [0, 1, 2, 3])
    bad = [
        (dict(layer=3, rows=ok), rg.RELAYGR_EINVAL), (dict(layer=-1, rows=ok), rg.RELAYGR_EINVAL), (dict(layer=0, rows=None), rg.RELAYGR_EINVAL),
        (dict(layer=0, rows=rg.KvRows(h, [1, 1, 2, 3])), rg.RELAYGR_EINVAL),                           # offsets that start behind 0
        (dict(layer=0, rows=rg.KvRows(h, [0, 2, 1, 3])), rg.RELAYGR_EINVAL),                           # or fall
        (dict(layer=0, rows=rg.KvRows(h, [0, 1, 2, 103])), rg.RELAYGR_EINVAL),                         # 101 tokens of 100
        (dict(layer=0, rows=rg.KvRows(h, [0, 1, 2, 3], first_token=[0, 0, 100])), rg.RELAYGR_EINVAL),
        (dict(layer=0, rows=rg.KvRows(h, [0, 1, 2, 3], first_token=[0, -1, 0])), rg.RELAYGR_EINVAL),
        (dict(layer=0, rows=rg.KvRows(h, [0, 1, 2, 3], first_token=[0, 2 ** 31 - 1, 0])), rg.RELAYGR_EINVAL),
        (dict(layer=0, rows=rg.KvRows([h[0], 0, h[2]], [0, 1, 2, 3])), rg.RELAYGR_ENOENT),
        (dict(layer=0, rows=rg.KvRows([h[0], h[1] + (1 << 32), h[2]], [0, 1, 2, 3])), rg.RELAYGR_ENOENT),
        (dict(layer=0, rows=ok, k=None), rg.RELAYGR_EINVAL), (dict(layer=0, rows=ok, v=None), rg.RELAYGR_EINVAL),
        (dict(layer=0, rows=ok, k=0x1008), rg.RELAYGR_EINVAL), (dict(layer=0, rows=ok, v=0x1002), rg.RELAYGR_EINVAL),
        (dict(layer=0, rows=ok, ks=260), rg.RELAYGR_EINVAL), (dict(layer=0, rows=ok, vs=248), rg.RELAYGR_EINVAL),
        (dict(layer=0, rows=ok, ks=-256), rg.RELAYGR_EINVAL),
    ]
    for kw, code in bad:
        rc, text = _call(p, name, **kw)
        assert rc == code and text, (kw, rc, text)
    same = rg.KvRows([h[0], h[1], h[0]], [0, 1, 2, 3], first_token=[0, 0, 64])
    if name == "relaygr_kv_pool_write":
        assert _call(p, name, 0, same)[0] == rg.RELAYGR_EINVAL
    # a pool of 16-bit K/V is another thing
    p16 = FakePool(cfg, q8=False)
    h16 = rg.relaygr_kv_pool_alloc(p16, 5, 100)
    assert _call(p16, name, 0, rg.KvRows([h16], [0, 1]))[0] == rg.RELAYGR_EINVAL
    # nothing to do is no error, whatever the arrays
    assert _call(p, name, 0, rg.KvRows([], [0]), k=None, v=None)[0] == 0
    assert _call(p, name, 0, rg.KvRows(h, [0, 0, 0, 0]), k=None, v=None)[0] == 0
    assert _call(p, name, 0, rg.KvRows([h[0], h[0]], [0, 0, 0]), k=None, v=None)[0] == 0


def test_attend_refuses_without_a_context_or_pool():
    lib = rg.load_library()
    cfg = rg.make_config(**CFG)
    p = FakePool(cfg)
    rows = rg.KvRows([rg.relaygr_kv_pool_alloc(p, 1, 100)], [0, 1])
    assert lib.relaygr_cache_attend(None, p.handle, 0, C.byref(rows.c), 0, 0x1000, 256, 0x2000, 256, None) == rg.RELAYGR_EINVAL
    assert "null" in rg.relaygr_last_error()


def test_binding_refuses_tensors_that_are_not_rows():
    cfg = rg.make_config(**CFG)
    p = FakePool(cfg)
    p.slab = torch.empty(1)     # (the binding asks it for its device)
    rows = rg.KvRows([rg.relaygr_kv_pool_alloc(p, 1, 100)], [0, 3])
    good = torch.zeros(3, 256, dtype=torch.bfloat16)
    assert B._kv_rows_array("x", p, rows, good) == (good.data_ptr(), 256)
    assert B._kv_rows_array("x", p, rows, good.view(3, 4, 64)) == (good.data_ptr(), 256)
    wide = torch.zeros(3, 1024, dtype=torch.bfloat16)
    assert B._kv_rows_array("x", p, rows, wide[:, 256:512]) == (wide.data_ptr() + 512, 1024)
    for t in (good[:2], good.half(), good.float(), torch.zeros(3, 128, dtype=torch.bfloat16), torch.zeros(256, 3, dtype=torch.bfloat16).T,
              torch.zeros(3, 2, 128, dtype=torch.bfloat16), torch.zeros(4, 3, 64, dtype=torch.bfloat16).transpose(0, 1), good[0], good.to("meta")):
        with pytest.raises(rg.RelayGRError) as e:
            B._kv_rows_array("x", p, rows, t)
        assert e.value.code == rg.RELAYGR_EINVAL
    for kw in (dict(row_off=[0, 1, 2]), dict(row_off=[0, 1], first_token=[0, 0]), dict(row_off=[0, 1], key_len=[])):
        with pytest.raises(rg.RelayGRError):
            rg.KvRows([1], **kw)


def test_the_reference_of_the_gpu_tests():
    """e4m3 against torch's cast, over all of its range; the scale against its two conditions."""
    x = np.concatenate([np.linspace(-448, 448, 20011), np.ldexp(np.linspace(-2, 2, 4099), -6), np.ldexp(np.linspace(-16, 16, 1025), -9)])
    x = x.astype(np.float32).astype(np.float64)
    want = torch.from_numpy(x).float().to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(e4m3(x), want)
    rng = np.random.default_rng(0)
    for top in list(np.exp(rng.uniform(-60, 60, 300))) + [1.75, 448.0, 1.75 * 2 ** -20, np.nextafter(1.75, 2)]:
        e = exponent(np.array([top, -top / 3]))
        assert top <= 448 * 2.0 ** e and (top > 448 * 2.0 ** (e - 1) or e == -100)
    assert exponent(np.zeros(3)) == -100 and exponent(np.array([np.nan, np.inf])) == -100
    y = held(np.array([1.0, -3.1, np.inf, np.nan, 1e-4]).reshape(5, 1, 1), "bf16").ravel()
    assert y[0] == 1.0 and y[1] == -3.0 and np.isnan(y[2:4]).all() and y[4] == 7 * 2.0 ** -16


def test_pieces_of_a_key_sequence():
    """Every key tile is in one piece, none is empty, and there are at most 64 of them."""
    for nk in list(range(0, 70)) + [127, 128, 129, 255, 256, 1000, 33554431]:
        for piece in (0, 1, 3, 4, 8, 100, 1 << 20):
            parts = rule_shim().attend_parts_of(nk, piece)
            per = max(1, -(-nk // parts))
            assert 1 <= parts <= 64 and (nk == 0 or (parts - 1) * per < nk <= parts * per)
            assert piece > 0 or parts == 1
    assert rule_shim().attend_parts_of(5, 4) == 1 and rule_shim().attend_parts_of(6, 4) == 2


def test_rule_of_the_attention_kernels():
    def rule(users, rows, keys, heads=8, dh=64):
        return attend_rule([rows] * users, [keys] * users, heads, dh)
    assert rule(16, 512, 4096) == {"blocks": 2, "once": 0, "piece": 0, "parts": 1}
    assert rule(16, 512, 4096, dh=128)["blocks"] == 1 and rule(16, 512, 4096, dh=32)["blocks"] == 1
    assert rule(64, 100, 4096)["blocks"] == 1 and rule(1, 512, 4096)["blocks"] == 1
    assert rule(128, 1, 8192)["once"] == 1 and rule(128, 33, 8192)["once"] == 0 and rule(8, 1, 8192)["once"] == 0
    assert rule(1, 1, 2048, heads=4)["parts"] == 8                       # four items: cut until the pieces are short
    assert rule(1, 512, 4096)["parts"] == 2                              # 128 items: one for each compute unit and no more
    assert rule(20, 20, 300)["parts"] == 1                               # too short to be worth a second launch
    long_one = attend_rule([30] * 32, [1000] * 31 + [16384], 8, 64)
    assert long_one["parts"] > 4 and attend_rule([30] * 32, [1000] * 32, 8, 64)["parts"] == 1
    assert attend_rule([5], [0], 8, 64)["parts"] == 1


def test_who_joins_the_pieces_of_few_users():
    joins = rule_shim().attend_joins
    joins.argtypes = [C.c_int, C.c_int64, C.c_int]
    assert joins(64, 512, 4096) == 1 and joins(256, 4096, 4096) == 1
    assert joins(257, 512, 4096) == 0                                    # many sums for one workgroup
    assert joins(64, 4097, 4096) == 0                                    # more items than counters
