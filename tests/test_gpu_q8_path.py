"""Pre-inference into an 8-bit pool and ranking on it.  What pre-inference leaves there is the definition's rounding of what it leaves in a 16-bit
pool, bit for bit; a ranking gives the same bits as one on a 16-bit pool that holds the values the codes stand for, whatever kernel it takes,
so that every test of the 16-bit path speaks for this one; and the scores are the oracle's on those values."""
import numpy as np
import pytest
import torch

import oracle
import paper_2601_01712_amd as rg
import plan_util
import synth
from gpu_util import BOOST, Harness, assert_close, build_case
from q8_util import held, offsets
from synth.generator import user_slices

pytestmark = pytest.mark.gpu


class Pair(Harness):
    """The same batch pre-inferred into an 8-bit pool and into a 16-bit one, which is then given the 8-bit pool's values."""

    def __init__(self, cfg, weights, batch, miss=()):
        super().__init__(cfg, weights, batch, 64)
        L = np.diff(batch["prefix_off"]).astype(int)
        self.users = [u for u in range(batch["n_users"]) if L[u] > 0 and u not in miss]
        self.prefill(self.users)
        self.lens = [int(L[u]) for u in self.users]
        pages = sum(-(-n // 64) for n in self.lens) + 2 + 4            # (room for one more of 200 tokens)
        self.pool8 = rg.KvPool(self.ctx.cfg, cfg.dtype, pages * rg.relaygr_kv_pool_bytes_for_q8(self.ctx.cfg, 64, 64), 64, quantized=True)
        self.pool8.slab.fill_(0x7F)
        rg.relaygr_kv_pool_alloc(self.pool8, 1 << 40, 65)              # (entries at other places than in the 16-bit pool)
        self.handles8 = np.zeros_like(self.handles)
        for u in self.users:
            self.handles8[u] = rg.relaygr_kv_pool_alloc(self.pool8, int(batch["user_ids"][u]), int(L[u]))
        sub = self.sub_batch(self.users)
        sub.set_handles([self.handles8[u] for u in self.users])
        rg.relaygr_prefill_prefix(self.ctx, self.pool8, sub)
        torch.cuda.synchronize()
        # where the 16-bit pool has its elements: one tile's pattern, and the strides
        d, first = cfg.d_model, self.handles[self.users[0]]
        at = np.array([[rg.relaygr_kv_pool_locate(self.pool, first, 0, r, f) for f in range(d)] for r in range(min(64, self.lens[0]))])
        if self.lens[0] < 64:
            longest = int(np.argmax(self.lens))
            assert self.lens[longest] >= 64
            first = self.handles[self.users[longest]]
            at = np.array([[rg.relaygr_kv_pool_locate(self.pool, first, 0, r, f) for f in range(d)] for r in range(64)])
        self.pattern = at - at[0, 0, 0]
        self.read8 = {l: [t.cpu() for t in rg.relaygr_kv_pool_read(self.pool8, l, rg.KvRows([self.handles8[u] for u in self.users], offsets(self.lens)))]
                      for l in range(cfg.n_layers)}

    def places(self, user, layer, n):
        """Indices [n, d, 2] of K and V of the user's tokens in the 16-bit slab."""
        base = [rg.relaygr_kv_pool_locate(self.pool, self.handles[user], layer, t, 0)[0] for t in range(0, n, 64)]
        return np.concatenate([b + self.pattern for b in base])[:n]

    def rank8(self):
        self.dbatch.set_handles(self.handles8)
        s = rg.relaygr_rank_with_cache(self.ctx, self.pool8, self.dbatch)
        torch.cuda.synchronize()
        return s.cpu().numpy()

    def check(self):
        cfg, heads, dh = self.cfg, self.cfg.n_heads, self.cfg.d_model // self.cfg.n_heads
        slab = self.pool.elements()
        at = offsets(self.lens)
        psi = {u: [] for u in self.users}
        for layer in range(cfg.n_layers):
            k8, v8 = self.read8[layer]
            for i, (u, n) in enumerate(zip(self.users, self.lens)):
                idx = torch.from_numpy(self.places(u, layer, n)).to(slab.device)
                for j, x8 in enumerate((k8[at[i]:at[i + 1]], v8[at[i]:at[i + 1]])):
                    x16 = slab[idx[..., j]].double().cpu().numpy()
                    assert np.array_equal(x8.double().numpy(), held(x16.reshape(n, heads, dh), cfg.dtype).reshape(n, -1)), (layer, u, "kv"[j])
                    slab[idx[..., j]] = x8.to(slab.device)
                psi[u].append((k8[at[i]:at[i + 1]].double(), v8[at[i]:at[i + 1]].double()))
        got, want = self.rank8(), self.rank_cached()
        assert np.isfinite(got).all() and np.array_equal(got, want)
        assert np.array_equal(self.rank8(), got)
        return got, psi

    def check_scores(self, got, psi):
        co = self.batch["cand_off"]
        for u in self.users:
            _, s, c = user_slices(self.batch, u)
            want = oracle.rank_with_kv(self.cfg, self.weights, psi[u], s, c)
            assert_close(got[co[u]:co[u + 1]], want, self.cfg.dtype, f"user {u}")

    def close(self):
        self.pool8.close()
        super().close()


#   d, heads, dtype, prefix lengths, suffix lengths, candidates, users without a cache
CASES = [
    (128, 4, "bf16", [100, 64, 65], [0, 3, 70], [10, 40, 5], ()),               # d_head 32
    (128, 2, "fp16", [1, 200, 63], [5, 0, 1], [1, 130, 33], ()),
    (256, 4, "bf16", [700, 300, 129, 0], [5, 0, 64, 9], [300, 130, 7, 20], (1,)),   # cached, recomputed and empty prefixes in one call
    (256, 2, "fp16", [500, 90], [3, 0], [64, 300], ()),                         # d_head 128
    (512, 8, "bf16", [1100], [0], [100], ()),                                   # cut into pieces
    (1024, 8, "bf16", [300, 70], [2, 0], [140, 33], (1,)),
]


@pytest.mark.parametrize("attention", ["silu", "softmax"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_same_bits_as_a_16_bit_pool_of_the_same_values(case, attention):
    d, heads, dtype, L, S, M, miss = CASES[case]
    cfg = synth.ModelConfig(2, d, heads, dtype, attention=attention)
    weights, batch = build_case(cfg, 9100 + case, L, S, M, boost=BOOST if d == 128 else None)
    h = Pair(cfg, weights, batch, miss)
    try:
        got, psi = h.check()
        h.check_scores(got, psi)
        out = torch.empty(len(got), dtype=torch.float32, device="cuda:0")
        h.dbatch.set_handles(h.handles8)
        rg.relaygr_rank_with_cache_static(h.ctx, h.pool8, h.dbatch, out)
        assert np.array_equal(out.cpu().numpy(), got)
    finally:
        h.close()


#   the kernels' other shapes: 128-row blocks of an item, wavefront groups, whether these share the pieces of a launch that the plan did not pair
SHAPES = [
    (512, 8, "bf16", [200] * 33, [0] * 33, [256] * 33, 2, 1, False),
    (512, 8, "fp16", [1300] * 16, [0, 5] * 8, [500] * 16, 2, 2, True),
    (512, 8, "bf16", [1100] * 20, [0, 70] * 10, [100] * 20, 1, 1, False),
    (512, 8, "bf16", [9000], [3], [509], 1, 1, True),
    (1024, 8, "bf16", [130] * 33, [3] * 33, [250] * 33, 2, 1, False),
    (256, 4, "fp16", [64, 1000, 250] * 30, [0] * 90, [256] * 90, 2, 1, False),
]


@pytest.mark.parametrize("attention", ["silu", "softmax"])
@pytest.mark.parametrize("case", range(len(SHAPES)))
def test_other_shapes_of_the_kernels(case, attention):
    d, heads, dtype, L, S, M, blocks, groups, shared = SHAPES[case]
    plan = plan_util.check(plan_util.shim(), L, S, M, [0] * len(L), heads, d // heads)
    least = plan_util.shared_pieces(attention, L, S, M, None, heads, d // heads)[1]
    assert (plan["blocks"], plan["gs"], least is not None) == (blocks, groups, shared)
    cfg = synth.ModelConfig(1, d, heads, dtype, attention=attention)
    weights, batch = build_case(cfg, 9300 + case, L, S, M)
    h = Pair(cfg, weights, batch)
    try:
        h.check()
    finally:
        h.close()


def test_batches_of_more_users_than_travel_in_the_kernels_arguments():
    cfg = synth.ModelConfig(2, 128, 2, "bf16")
    rng = np.random.default_rng(2)
    n = 150
    L = [int(x) for x in rng.integers(1, 200, n)]
    L[0] = 64
    weights, batch = build_case(cfg, 9401, L, [int(x) for x in rng.integers(0, 3, n)], [int(x) for x in rng.integers(1, 9, n)], boost=BOOST)
    h = Pair(cfg, weights, batch)
    try:
        h.check_scores(*h.check())
    finally:
        h.close()


def test_appended_behaviours_join_a_pre_inferred_prefix():
    """Most of a history written in one call and its last tokens' K and V one by one: the entry then ranks like the one that pre-inference left."""
    cfg = synth.ModelConfig(2, 256, 4, "bf16")
    weights, batch = build_case(cfg, 9501, [200], [0], [50])
    h = Pair(cfg, weights, batch)
    try:
        whole = {l: h.read8[l] for l in range(2)}
        grown = rg.relaygr_kv_pool_alloc(h.pool8, 4242, 200)
        for l in range(2):
            k, v = (t.cuda() for t in whole[l])
            rg.relaygr_kv_pool_write(h.pool8, l, rg.KvRows([grown], [0, 130]), k[:130], v[:130])
            for t in range(130, 200):
                rg.relaygr_kv_pool_write(h.pool8, l, rg.KvRows([grown], [0, 1], first_token=[t]), k[t:t + 1], v[t:t + 1])
            # (values that are codes already: as a block's scale grows with its tokens none of them is smaller than the final scale's steps)
            got = [t.double().cpu().numpy() for t in rg.relaygr_kv_pool_read(h.pool8, l, rg.KvRows([grown], [0, 200]))]
            for g, w in zip(got, whole[l]):
                assert np.array_equal(g, w.double().numpy())
        want = h.rank8()
        h.handles8[0] = grown
        assert np.array_equal(h.rank8(), want)
    finally:
        h.close()


def test_context_and_pool_of_different_shapes_are_refused():
    cfg = synth.ModelConfig(2, 128, 2, "bf16")
    weights, batch = build_case(cfg, 9601, [70], [0], [5])
    h = Harness(cfg, weights, batch)
    try:
        other = rg.make_config(2, 128, 4, "bf16")
        pool = rg.KvPool(other, "bf16", 4 * rg.relaygr_kv_pool_bytes_for_q8(other, 64, 64), 64, quantized=True)
        handle = rg.relaygr_kv_pool_alloc(pool, 1, 70)
        h.dbatch.set_handles([handle])
        for call in (lambda: rg.relaygr_prefill_prefix(h.ctx, pool, h.dbatch), lambda: rg.relaygr_rank_with_cache(h.ctx, pool, h.dbatch)):
            with pytest.raises(rg.RelayGRError) as e:
                call()
            assert e.value.code == rg.RELAYGR_EINVAL
    finally:
        h.close()
