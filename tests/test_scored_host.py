"""Refusals of scored attention and eviction that need no GPU: nothing here gets as far as a launch, and the slab's address is never dereferenced."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
from paper_2601_01712_amd import binding as B
from scored_util import scored, visible
from test_q8_host import CFG, FakePool


def eviction(**kw):
    e = dict(first=0, recent=0, weight=0x100000, position=0x200000, token_off=[0, 1000, 2000], kept=0x300000, weight_out=0x400000, position_out=0x500000, out_off=None, to=None) | kw
    keep = []

    def ptr(x, dtype):
        if x is None:
            return None
        keep.append(np.array(x, dtype=dtype))
        return keep[-1].ctypes.data
    c = B.KvEvictionC(e["first"], e["recent"], ptr(e["to"], np.uint64), e["weight"], e["position"], ptr(e["token_off"], np.int64), e["kept"], e["weight_out"],
                      e["position_out"], ptr(e["out_off"], np.int64))
    c.keep = keep
    return c


def test_eviction_refuses():
    lib, p = rg.load_library(), FakePool(rg.make_config(**CFG), pages=20)
    h = [rg.relaygr_kv_pool_alloc(p, u, 100) for u in range(3)]
    to = [rg.relaygr_kv_pool_alloc(p, 10 + u, 64) for u in range(3)]

    def call(rows=None, e=None, pool=p.handle, **kw):
        rows = rg.KvRows(h, [0, 50, 100, 150], key_len=[100, 90, 80]) if rows is None else rows
        return lib.relaygr_kv_pool_evict(pool, rows.ref, C.byref(eviction(**kw) if e is None else e), None)
    cases = [
        (dict(rows=rg.KvRows(h, [0, 50, 100, 181], key_len=[100, 90, 80])), rg.RELAYGR_EINVAL), (dict(rows=rg.KvRows(h, [0, 50, 100, 150], key_len=[100, 101, 80])), rg.RELAYGR_EINVAL),
        (dict(rows=rg.KvRows(h, [0, 50, 100, 150], key_len=[100, -1, 80])), rg.RELAYGR_EINVAL), (dict(rows=rg.KvRows(h, [1, 50, 100, 150])), rg.RELAYGR_EINVAL),
        (dict(rows=rg.KvRows(h, [0, 50, 40, 150])), rg.RELAYGR_EINVAL), (dict(rows=rg.KvRows([h[0], 0, h[2]], [0, 50, 100, 150])), rg.RELAYGR_ENOENT),
        (dict(rows=rg.KvRows([h[0], h[1], h[0]], [0, 50, 100, 150])), rg.RELAYGR_EINVAL), (dict(first=-1), rg.RELAYGR_EINVAL), (dict(recent=-1), rg.RELAYGR_EINVAL),
        (dict(first=25, recent=26), rg.RELAYGR_EINVAL), (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), rg.RELAYGR_EINVAL), (dict(weight=None), rg.RELAYGR_EINVAL), (dict(kept=None), rg.RELAYGR_EINVAL),
        (dict(token_off=None), rg.RELAYGR_EINVAL), (dict(weight=0x100002), rg.RELAYGR_EINVAL), (dict(kept=0x300001), rg.RELAYGR_EINVAL), (dict(position=None), rg.RELAYGR_EINVAL),
        (dict(token_off=[0, -1, 2000]), rg.RELAYGR_EINVAL), (dict(out_off=[0, 50, -100]), rg.RELAYGR_EINVAL), (dict(out_off=[0, 49, 100]), rg.RELAYGR_EINVAL), (dict(to=[to[0], to[1], to[1]]), rg.RELAYGR_EINVAL),
        (dict(to=[to[0], to[1], 99]), rg.RELAYGR_ENOENT), (dict(to=[to[0], h[0], to[2]]), rg.RELAYGR_EINVAL), (dict(rows=rg.KvRows(h, [0, 65, 100, 150]), to=to), rg.RELAYGR_EINVAL),
        # outputs over inputs: only a user's own, from the same element on, and only if the inputs are nobody else's
        (dict(weight_out=0x100000, out_off=[4, 1000, 2000]), rg.RELAYGR_EINVAL), (dict(weight_out=0x100000, out_off=[1000, 0, 2000]), rg.RELAYGR_EINVAL),
        (dict(weight_out=0x100000, token_off=[0, 0, 2000], out_off=[0, 1000, 2000]), rg.RELAYGR_EINVAL), (dict(position_out=0x200000 + 396, out_off=[0, 1000, 2000]), rg.RELAYGR_EINVAL),
    ]
    for kw, code in cases:
        rc = call(**kw)
        assert rc == code and rg.relaygr_last_error(), (kw, rc, rg.relaygr_last_error())
    assert call(pool=None) == rg.RELAYGR_EINVAL
    assert lib.relaygr_kv_pool_evict(p.handle, None, C.byref(eviction()), None) == rg.RELAYGR_EINVAL
    assert lib.relaygr_kv_pool_evict(p.handle, rg.KvRows(h, [0, 1, 2, 3]).ref, None, None) == rg.RELAYGR_EINVAL
    p16 = FakePool(rg.make_config(**CFG), q8=False)
    assert call(pool=p16.handle, rows=rg.KvRows([rg.relaygr_kv_pool_alloc(p16, 5, 100)], [0, 1])) == rg.RELAYGR_EINVAL
    # nothing stays anywhere, or there is nobody: no error, whatever the arrays
    assert call(rows=rg.KvRows(h, [0, 0, 0, 0]), weight=None, kept=None, position=None, position_out=None, token_off=None) == 0
    assert call(rows=rg.KvRows([], [0]), weight=None, kept=None) == 0


def test_scored_attention_refuses_without_a_context_or_pool():
    lib, p = rg.load_library(), FakePool(rg.make_config(**CFG))
    rows, s = rg.KvRows([rg.relaygr_kv_pool_alloc(p, 1, 100)], [0, 1]), rg.Scoring(cap=1.0)
    assert lib.relaygr_cache_attend_scored(None, p.handle, 0, rows.ref, 0, s.ref, 0x1000, 256, 0x2000, 256, None, None, None) == rg.RELAYGR_EINVAL
    assert "null" in rg.relaygr_last_error()


def test_the_reference_of_the_gpu_tests():
    """Masks by their words, and the formula against loops."""
    see = visible(6, 3, causal=True, prefix=2, window=2)
    assert see.astype(int).tolist() == [[1, 1, 1, 1, 0, 0], [1, 1, 0, 1, 1, 0], [1, 1, 0, 0, 1, 1]]
    assert not visible(4, 2, first=np.array([4, 3]), end=np.array([9, 0])).any()
    assert visible(3, 5, causal=True).sum(axis=1).tolist() == [0, 0, 1, 2, 3]
    rng = np.random.default_rng(0)
    q, k, v = rng.standard_normal((2, 2, 4)), rng.standard_normal((5, 2, 4)), rng.standard_normal((5, 2, 4))
    slopes, rp, kp = np.array([0.5, 0.25]), np.array([9, 11]), np.array([0, 2, 5, 6, 20])
    for form in ("softmax", "silu"):
        see = visible(5, 2, first=np.array([1, 0]), end=np.array([4, 5]))
        out, _, total, _ = scored(q, k, v, see, form, "bf16", 1.5, slopes, rp, kp)
        sums = np.zeros(5)
        for i in range(2):
            for h in range(2):
                w = np.zeros(5)
                for j in range(5):
                    if not see[i, j]:
                        continue
                    s = sum(q[i, h, f] * k[j, h, f] for f in range(4)) / 2.0
                    s = 1.5 * np.tanh(s / 1.5) - slopes[h] * abs(float(rp[i]) - float(kp[j]))
                    w[j] = np.exp(s) if form == "softmax" else s / (1 + np.exp(-s)) / see[i].sum()
                if form == "softmax":
                    w /= w.sum()
                sums += np.abs(w)
                assert np.allclose(out[i, h], w @ v[:, h], rtol=1e-12, atol=1e-14)
        assert np.allclose(total, sums, rtol=1e-12)


@pytest.mark.parametrize("kw", [dict(prefix=[[1, 2]]), dict(token_off=[[0]])])
def test_host_arrays_are_vectors(kw):
    with pytest.raises(rg.RelayGRError):
        rg.Scoring(**kw)


def test_scoring_is_what_it_was_made_with():
    s = rg.Scoring(cap=2.0, prefix=[1, 2], token_off=[0, 10])
    for name, value in (("prefix", [3, 4]), ("row_first", None if s.row_first is not None else np.zeros(2)), ("window", 5)):
        with pytest.raises(AttributeError):
            setattr(s, name, value)
    s.prefix[:] = 7
    s.token_off += 1
    assert list(s.c.prefix[:2]) == [7, 7] and list(s.c.token_off[:2]) == [1, 11]


@pytest.mark.parametrize("kw", [dict(cap=1e-50), dict(cap=-1e-50), dict(window=2 ** 32), dict(window=2 ** 31), dict(window=2 ** 32 + 5), dict(window=-2 ** 31 - 1), dict(prefix=np.array([2 ** 32 + 3])),
                                dict(prefix=np.array([1, -2 ** 32])), dict(prefix=[2 ** 40]), dict(prefix=[5, 2 ** 70]), dict(prefix=np.array([2 ** 32 - 1], np.uint32))])
def test_numbers_that_the_struct_would_hold_as_others_are_refused(kw):
    with pytest.raises(rg.RelayGRError) as e:
        rg.Scoring(**kw)
    assert e.value.code == rg.RELAYGR_EINVAL


def test_numbers_at_the_ends_of_their_types():
    s = rg.Scoring(cap=2.0 ** -100, window=2 ** 31 - 1, prefix=np.array([2 ** 31 - 1, 0]))
    assert s.c.cap == 2.0 ** -100 and s.c.window == 2 ** 31 - 1 and s.prefix.tolist() == [2 ** 31 - 1, 0]
    assert rg.Scoring(prefix=[]).prefix.size == 0


@pytest.mark.parametrize("kw", [dict(first=2 ** 32), dict(recent=2 ** 32 + 4), dict(first=-2 ** 32), dict(recent=2 ** 31)])
def test_eviction_refuses_counts_beyond_their_type(monkeypatch, kw):
    p = FakePool(rg.make_config(**CFG), pages=20)
    p.slab = torch.zeros(0)
    monkeypatch.setattr(B, "_kv_guard", lambda pool, stream: None)
    with pytest.raises(rg.RelayGRError, match="beyond 32 bits"):
        rg.relaygr_kv_pool_evict(p, rg.KvRows([rg.relaygr_kv_pool_alloc(p, 1, 100)], [0, 10], key_len=[100]), torch.zeros(100), [0], **kw)


@pytest.mark.parametrize("cap", [2.0 ** -100, 1.0, 30.0, 50.0, 128.0])
def test_the_bound_of_capped_scores(cap):
    """cap - 2 cap / (1 + exp(2 t / cap)) in 32 bits, with exp2 and the reciprocal off by an ulp either way: within 4.3 * 2^-23 of the cap."""
    rng, f, per_ln2 = np.random.default_rng(0), np.float32, 1.4426950408889634
    mul, add, cap_mul = f(-2 * cap * per_ln2), f(cap * per_ln2), f(2 * per_ln2 / cap)
    t = (np.concatenate([rng.uniform(-12, 12, 50000), rng.uniform(-2, 2, 50000), np.exp(rng.uniform(-20, 3, 20000))]) * cap / 2).astype(f)
    want = cap * np.tanh(t.astype(np.float64) / cap) * per_ln2
    for exp_off in (0, 1, -1):
        for rcp_off in (0, 1, -1):
            e = np.exp2((t * cap_mul).astype(np.float64)).astype(f)
            e = np.nextafter(e, f(exp_off * np.inf)) if exp_off else e
            r = (1.0 / (f(1) + e).astype(np.float64)).astype(f)
            r = np.nextafter(r, f(rcp_off * np.inf)) if rcp_off else r
            got = (mul.astype(np.float64) * r + add).astype(f)
            assert np.abs(got - want).max() <= 4.3 * 2.0 ** -23 * cap * per_ln2
