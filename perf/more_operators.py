"""Performance cases of what a backbone with its own projections does around an 8-bit K/V cache besides writing it: positions, scored attention, eviction.

Three calls: `rotate` (relaygr_rotary: rotary positions of rows of q, or of q and k), `attend` (relaygr_cache_attend_scored: query rows over the cached
keys with scores that are capped or get a bias that falls with the distance, and with masks; where asked, with the weight that each cached token
received added up) and `evict` (relaygr_kv_pool_evict: the tokens with the least of that weight leave their entries).  A case
names the call, the width, heads and storage type, and its batch.  rotate:

    rows                 rows of q (and of k, with `both`)
    far                  positions are uniform in [0, far)
    dim, layout          features of a head that are rotated; "half" or "interleaved" pairs
    factor, original     frequencies are divided by `factor`: all of them (original 0), or those that turn seldom in `original` positions
    transposed           the rotation back, which is the gradient's

attend and evict:

    users                users in the call
    keys, keys_sigma     tokens of the entries: all `keys` (sigma 0), or lognormal around it with that sigma, clipped to [1, 16384]
    rows_lo, rows_hi     attend: query rows a user, uniform in the range
    causal               attend: the rows are the last of the keys, each sees those up to its own
    cap, bias            attend: 0 or the cap of the scores; slopes by the heads, times the distance
    gaps                 attend: positions of the keys that are not their places in the entry (some left it before)
    session              attend: 0, or the mean length of the sessions that a history is of: rows see their own session
    prefix               attend: tokens at the front of every entry that all rows see
    window               attend: 0, or how many tokens up to its own a row sees
    weigh                attend: whether the tokens' weights are added up
    keep                 evict: share of a user's tokens that stay
    first, recent        evict: tokens at the front and at the end that stay whatever their weight
    shape_seed           seed of lengths, sessions and kept counts, which belong to the case; the values belong to prepare()'s seed
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 64              # tokens that share a scale
LAYERS, LAYER = 2, 1    # of the pool, and the one that attention is for
PAGE_TOKENS = 256
BASE = 10000.0
TURNS_LOW, TURNS_HIGH = 1.0, 32.0     # turns in `original` positions: below the first fully divided, above the second as they are
_TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _rotate(d, heads, dtype, rows, far, dim, layout="half", both=True, factor=1.0, original=0, transposed=False):
    return {"call": "rotate", "d": d, "heads": heads, "dtype": dtype, "rows": rows, "far": far, "dim": dim, "layout": layout, "both": both,
            "factor": factor, "original": original, "transposed": transposed}


def _attend(d, heads, dtype, form, users, keys, rows, keys_sigma=0.0, causal=False, cap=0.0, bias=False, gaps=False, session=0, prefix=0, window=0,
            weigh=False, shape_seed=0):
    return {"call": "attend", "d": d, "heads": heads, "dtype": dtype, "form": form, "users": users, "keys": keys, "keys_sigma": keys_sigma,
            "rows_lo": rows[0], "rows_hi": rows[1], "causal": causal, "cap": cap, "bias": bias, "gaps": gaps, "session": session, "prefix": prefix,
            "window": window, "weigh": weigh, "shape_seed": shape_seed}


def _evict(d, heads, dtype, users, keys, keep, first, recent, keys_sigma=0.0, shape_seed=0):
    return {"call": "evict", "d": d, "heads": heads, "dtype": dtype, "users": users, "keys": keys, "keys_sigma": keys_sigma, "keep": keep, "first": first,
            "recent": recent, "shape_seed": shape_seed}


def listed():
    cases = {
        # one new behaviour's q and k: a launch and little else
        "rotate_one_row": _rotate(256, 4, "bf16", 1, 5000, 64),
        # a chunk of behaviours of a model that rotates half of each head, stretched to eight times the length it was made for
        "rotate_part_of_head": _rotate(512, 8, "fp16", 4701, 1 << 20, 32, "interleaved", factor=8.0),
        # whole histories of a batch of users, before they are written
        "rotate_histories": _rotate(512, 8, "bf16", 65536, 16384, 64, factor=4.0, original=4096),
        # a projection's gradient on its way back through the rotation
        "rotate_gradient": _rotate(1024, 8, "fp32", 8192, 8192, 128, both=False, transposed=True),
        # one new behaviour over a short history with capped scores: the latency of one layer
        "attend_step": _attend(256, 4, "bf16", "softmax", 1, 2048, (1, 1), cap=30.0),
        # one new behaviour each of many long histories, recent ones favoured, and what each cached token was worth
        "attend_steps_weighed": _attend(512, 8, "bf16", "softmax", 128, 8192, (1, 1), bias=True, weigh=True),
        # a chunk of new behaviours, each seeing the user's profile and its own session
        "attend_sessions": _attend(256, 8, "fp16", "softmax", 8, 2100, (100, 300), causal=True, cap=30.0, session=400, prefix=70, shape_seed=2),
        # a ranking's candidates over histories that have lost tokens before, pointwise form
        "attend_candidates": _attend(512, 8, "bf16", "silu", 16, 4096, (512, 512), bias=True, gaps=True),
        # the wide end of the embedding axis, sliding window
        "attend_window": _attend(1024, 8, "fp16", "softmax", 16, 8192, (200, 200), causal=True, cap=50.0, window=2000, prefix=16),
        # long ragged histories, many rows, everything at once (the largest case)
        "attend_ragged": _attend(512, 8, "bf16", "softmax", 32, 4096, (200, 1000), keys_sigma=0.7, cap=30.0, bias=True, weigh=True, shape_seed=9),
        # one user's entry is full
        "evict_one_user": _evict(256, 4, "fp16", 1, 4095, 0.5, 4, 256),
        # a batch's entries go back to three quarters
        "evict_batch": _evict(512, 8, "bf16", 32, 4096, 0.75, 4, 64, keys_sigma=0.7, shape_seed=4),
    }
    return [dict(c, name=name) for name, c in cases.items()]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        call = rng.choice(["rotate", "attend", "attend", "attend", "evict"])
        d, heads = rng.choice([(128, 4), (256, 4), (256, 8), (512, 8), (512, 8), (1024, 8)])
        dtype, users, sigma, shape_seed = rng.choice(["bf16", "bf16", "fp16"]), _log_int(rng, 1, 128), rng.choice([0.0, 0.7]), rng.randrange(1 << 20)
        if call == "rotate":
            dh = d // heads
            factor = rng.choice([1.0, 4.0, 8.0])
            case = _rotate(d, heads, rng.choice(["fp32", dtype, dtype]), _log_int(rng, 1, 1 << 17), _log_int(rng, 100, 1 << 24), rng.choice([dh, dh // 2, 2 * rng.randint(1, dh // 2)]),
                           rng.choice(["half", "interleaved"]), rng.random() < 0.7, factor, rng.choice([0, 4096]) if factor > 1 else 0, rng.random() < 0.3)
        elif call == "attend":
            m = rng.choice([1, _log_int(rng, 1, 32), _log_int(rng, 32, 1024)])
            n = _log_int(rng, 16, 16384)
            causal = rng.random() < 0.5
            mask = rng.choice(["none", "none", "session", "window"])
            case = _attend(d, heads, dtype, rng.choice(["silu", "softmax", "softmax"]), users, n, (max(1, m // 3), m), sigma, causal, rng.choice([0.0, 0.0, 30.0, 50.0]),
                           rng.random() < 0.5, rng.random() < 0.3, _log_int(rng, 10, 2000) if mask == "session" else 0, rng.choice([0, 0, _log_int(rng, 1, 200)]),
                           _log_int(rng, 16, 4096) if mask == "window" else 0, rng.random() < 0.4, shape_seed)
        else:
            case = _evict(d, heads, dtype, users, _log_int(rng, 16, 16384), rng.choice([0.25, 0.5, 0.75, rng.uniform(0.05, 0.95)]), rng.choice([0, 4]), rng.choice([0, 1, 64, 256]),
                          sigma, shape_seed)
        if _cost(case) <= most and (call != "attend" or _padded(case) <= 1 << 32):
            return case


# ---- the batch: functions of the case alone ------------------------------------------------------------------------------
def _keys(case, r):
    out = []
    for _ in range(case["users"]):
        n = case["keys"]
        if case["keys_sigma"] > 0:
            n = min(16384, max(1, int(round(math.exp(r.gauss(math.log(n), case["keys_sigma"]))))))
        out.append(n)
    return out


def _lengths(case):
    r = random.Random(case["shape_seed"])
    keys = _keys(case, r)
    return keys, [r.randint(case["rows_lo"], case["rows_hi"]) for _ in keys]


def _evict_lengths(case):
    """Tokens of the entries, and how many of them stay (at least those that stay whatever their weight, if there are that many)."""
    keys = _keys(case, random.Random(case["shape_seed"]))
    return keys, [min(n, max(1, round(n * case["keep"]), case["first"] + case["recent"])) for n in keys]


def _ranges(case):
    """Of every row: the first and the end of the tokens that it sees behind the prefix, and the prefix; [rows] each."""
    keys, rows = _lengths(case)
    r = random.Random(case["shape_seed"] + 1)
    first, end, prefix = [], [], []
    for n, m in zip(keys, rows):
        e = np.clip(n - m + 1 + np.arange(m), 0, n) if case["causal"] else np.full(m, n)
        f = np.zeros(m, np.int64)
        if case["session"]:
            starts = [0]
            while starts[-1] < n:
                starts.append(starts[-1] + max(1, int(r.expovariate(1.0 / case["session"]))))
            starts = np.asarray(starts[:-1])
            f = starts[np.maximum(np.searchsorted(starts, np.maximum(e - 1, 0), side="right") - 1, 0)]
        if case["window"]:
            f = np.maximum(f, e - case["window"])
        p = min(case["prefix"], n)
        f = np.maximum(f, p)
        first.append(f)
        end.append(np.maximum(e, f))
        prefix.append(np.full(m, p))
    return [np.concatenate(x).astype(np.int64) for x in (first, end, prefix)]


def _blocks(n):
    return -(-n // BLOCK)


def _offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)


def _padded(case):
    """Scores of the padded batch, which the plain form holds at once."""
    keys, rows = _lengths(case)
    return case["users"] * case["heads"] * max(keys) * max(rows)


def work(case):
    d, heads = case["d"], case["heads"]
    scale = 4 * heads       # of a block of all heads of K or V
    if case["call"] == "rotate":
        e = _TORCH[case["dtype"]].itemsize
        elements = case["rows"] * d * (2 if case["both"] else 1)
        return {"bytes": 2 * e * elements + 4 * case["rows"], "flops": 3 * elements * case["dim"] // (d // heads)}
    if case["call"] == "evict":
        # all layers in and out, what is held of them read back, and the tokens' weights, positions and places
        keys, keep = _evict_lengths(case)
        moved = sum(2 * (d * n + scale * _blocks(n)) for n in keys) + 2 * sum(2 * (d * m + scale * _blocks(m)) for m in keep) + sum(4 * d * m for m in keep)
        return {"bytes": LAYERS * moved + 8 * sum(keys) + 12 * sum(keep), "flops": 0}
    keys, rows = _lengths(case)
    first, end, prefix = _ranges(case)
    ro = _offsets(rows)
    read = pairs = 0
    for u, n in enumerate(keys):
        f, e, p = (x[ro[u]:ro[u + 1]] for x in (first, end, prefix))
        pairs += int((p + e - f).sum())
        seen = np.zeros(n + 1, np.int64)         # tokens that any row sees
        np.add.at(seen, f, 1)
        np.add.at(seen, e, -1)
        read += int((((np.cumsum(seen)[:n]) > 0) | (np.arange(n) < p[0])).sum())
    total = 2 * (d + scale / BLOCK) * read + 4 * d * sum(rows) + (8 * sum(keys) if case["weigh"] else 0) + (4 * sum(keys) if case["gaps"] else 0)
    return {"bytes": int(total), "flops": 4 * d * pairs}


def _cost(case):
    w = work(case)
    return w["flops"] / 5e14 + w["bytes"] / 4e12


# ---- the quantisation in plain form ------------------------------------------------------------------------------------
def _exponent(amax):
    """Of the power-of-two scale of blocks whose largest magnitude is amax: amax / 2^e is the largest in e4m3's range that is at most 448."""
    m, x = torch.frexp(amax)                                # amax = m * 2^x, m in [0.5, 1)
    return torch.where(amax > 0, x - 9 + (m > 0.875).to(x.dtype), torch.full_like(x, -100)).clamp(min=-100)


def _pow2(e):
    """2^e in fp32 from its bits."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _quantise(x):
    """x [blocks, BLOCK, heads, dh] in fp32: e4m3 codes of that shape and the blocks' exponents [blocks, heads]."""
    e = _exponent(x.abs().amax(dim=(1, 3)))
    codes = (x * _pow2(-e)[:, None, :, None]).to(torch.float8_e4m3fn)
    return codes, e


def _dequantise(codes, e):
    return codes.float() * _pow2(e)[:, None, :, None]


def _in_blocks(lens):
    """Where each token of users of these lengths stands in their blocks' [blocks * BLOCK] places."""
    first = _offsets([_blocks(n) for n in lens]) * BLOCK
    return np.concatenate([np.arange(f, f + n) for f, n in zip(first, lens)] + [np.zeros(0, np.int64)])


def _gpu(a, dtype=np.int64):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=dtype)).to("cuda:0")


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _frequencies(case):
    """Radians a position of every pair, in 64 bits."""
    i = torch.arange(case["dim"] // 2, dtype=torch.float64)
    f = BASE ** (-2.0 * i / case["dim"])
    keep = ((f * case["original"] / (2 * math.pi) - TURNS_LOW) / (TURNS_HIGH - TURNS_LOW)).clamp(0.0, 1.0) if case["original"] else torch.zeros_like(f)
    return f * (keep + (1.0 - keep) / case["factor"])


def _gain(case):
    """What a stretched model multiplies its rotated features with: sharper scores over more tokens."""
    return 0.1 * math.log(case["factor"]) + 1.0 if case["original"] else 1.0


def _rows(gen, n, d, gain, dtype):
    """n rows as a layer's projection leaves them: SiLU of normal values whose features differ in size."""
    x = torch.randn((n, d), generator=gen, device="cuda:0") * gain
    return (x * torch.sigmoid(x)).to(dtype)


def _inputs(case, seed):
    """The values a case is made of, rows in the storage type."""
    gen = torch.Generator(device="cuda:0")
    gen.manual_seed(seed)
    d, dtype = case["d"], _TORCH[case["dtype"]]
    gain = [torch.exp(0.5 * torch.randn(d, generator=gen, device="cuda:0")) for _ in range(3)]
    if case["call"] == "rotate":
        out = {"pos": torch.randint(0, case["far"], (case["rows"],), generator=gen, device="cuda:0", dtype=torch.int32), "q": _rows(gen, case["rows"], d, gain[0], dtype)}
        if case["both"]:
            out["k"] = _rows(gen, case["rows"], d, gain[1], dtype)
        return out
    if case["call"] == "evict":
        keys, _ = _evict_lengths(case)
        out = {name + str(layer): _rows(gen, sum(keys), d, gain[i], dtype) for layer in range(LAYERS) for i, name in enumerate("kv")}
        # weights over several orders of magnitude; a tenth of the tokens were never looked at
        w = torch.exp(2.0 * torch.randn(sum(keys), generator=gen, device="cuda:0"))
        out["weight"] = torch.where(torch.rand(sum(keys), generator=gen, device="cuda:0") < 0.1, 0.0, w)
        out["pos"] = _climb(gen, keys)
        return out
    keys, rows = _lengths(case)
    out = {"k": _rows(gen, sum(keys), d, gain[0], dtype), "v": _rows(gen, sum(keys), d, gain[1], dtype), "q": _rows(gen, sum(rows), d, gain[2], dtype)}
    ro = _offsets(rows)
    last = np.concatenate([n - m + np.arange(m) if case["causal"] else np.full(m, n) for n, m in zip(keys, rows)])     # rows' places in their histories
    if case["gaps"]:
        out["key_pos"] = _climb(gen, keys)
        top = out["key_pos"][_gpu(_offsets(keys)[1:] - 1)].long()
        of_row = np.repeat(np.arange(len(rows)), rows)
        out["row_pos"] = (top[_gpu(of_row)] + 1 + _gpu(np.arange(ro[-1]) - ro[of_row])).int()
    else:
        out["key_pos"] = _gpu(np.concatenate([np.arange(n) for n in keys])).int()
        out["row_pos"] = _gpu(last).int()
    if case["weigh"]:
        out["weight"] = torch.rand(sum(keys), generator=gen, device="cuda:0")
    return out


def _climb(gen, lens):
    """Climbing positions for users of these lengths, from 0 on, about every second one missing."""
    step = torch.randint(1, 4, (sum(lens),), generator=gen, device="cuda:0")
    total = torch.cumsum(step, 0)
    first = _gpu(np.repeat(_offsets(lens)[:-1], lens))
    return (total - total[first]).int()


def _slopes(case):
    return torch.pow(2.0, -10.0 * (1.0 + torch.arange(case["heads"], dtype=torch.float64)) / case["heads"])


def prepare(case, seed):
    state = dict(_inputs(case, seed), case=case)
    d, heads = case["d"], case["heads"]
    dh = d // heads
    if own:
        import paper_2601_01712_amd as rg
        cfg = rg.make_config(LAYERS, d, heads, case["dtype"])
    if case["call"] == "rotate":
        state["freq"] = _frequencies(case).to("cuda:0")
        if own:
            state["cfg"] = cfg
            state["rope"] = rg.Rope(case["dim"], BASE, case["layout"], factor=case["factor"], original_len=case["original"], low=TURNS_LOW, high=TURNS_HIGH, gain=_gain(case))
        return state
    keys, other = _evict_lengths(case) if case["call"] == "evict" else _lengths(case)
    places = _gpu(_in_blocks(keys))
    state["held"] = places
    blocks = sum(_blocks(n) for n in keys)
    names = [n + str(layer) for layer in range(LAYERS) for n in "kv"] if case["call"] == "evict" else ["k", "v"]
    for name in names:
        x = torch.zeros((blocks * BLOCK, d), device="cuda:0")
        x[places] = state.pop(name).float()
        state[name + "_codes"], state[name + "_exp"] = _quantise(x.view(-1, BLOCK, heads, dh))
    if own:
        pool_bytes = sum(rg.relaygr_kv_pool_bytes_for_q8(cfg, n, PAGE_TOKENS) for n in keys)
        if case["call"] == "evict":
            pool_bytes += sum(rg.relaygr_kv_pool_bytes_for_q8(cfg, n, PAGE_TOKENS) for n in other)
        pool = state["pool"] = rg.KvPool(cfg, case["dtype"], pool_bytes, PAGE_TOKENS, quantized=True)
        handles = [rg.relaygr_kv_pool_alloc(pool, 1000 + u, n) for u, n in enumerate(keys)]
        whole = rg.KvRows(handles, _offsets(keys))
        for layer, (kn, vn) in [(i, ("k%d" % i, "v%d" % i)) for i in range(LAYERS)] if case["call"] == "evict" else [(LAYER, ("k", "v"))]:
            k, v = (_dequantise(state[n + "_codes"], state[n + "_exp"]).view(-1, d)[places].to(_TORCH[case["dtype"]]) for n in (kn, vn))
            rg.relaygr_kv_pool_write(pool, layer, whole, k, v)
        torch.cuda.synchronize()
    if case["call"] == "evict":
        # padded batch: which token stands where, which must stay, and where what stays goes
        L, M, tokens = max(keys), max(other), sum(keys)
        ko, at, kn, mn = _offsets(keys)[:-1, None], np.arange(L)[None], np.asarray(keys)[:, None], np.asarray(other)[:, None]
        state["at"] = _gpu(np.where(at < kn, ko + at, tokens))
        state["must"] = _gpu(((at < case["first"]) | (at >= kn - case["recent"])) & (at < kn), bool)
        state["stay"] = _gpu(np.arange(M)[None] < mn, bool)
        state["back"] = _gpu(np.concatenate([u * M + np.arange(m) for u, m in enumerate(other)]))
        state["token0"] = _gpu(np.repeat(_offsets(keys)[:-1], other))
        state["to"] = _gpu(_in_blocks(other))
        if own:
            to = [rg.relaygr_kv_pool_alloc(pool, 500000 + u, m) for u, m in enumerate(other)]
            state["rows"] = rg.KvRows(handles, _offsets(other), key_len=keys)
            state["read"] = rg.KvRows(to, _offsets(other))
            state["handles"] = np.asarray(to, np.uint64)
            state["token_off"] = _offsets(keys)[:-1]
            state["kept"] = torch.empty(sum(other), dtype=torch.int32, device="cuda:0")
            state["weight_out"] = torch.empty(sum(other), device="cuda:0")
            state["pos_out"] = torch.empty(sum(other), dtype=torch.int32, device="cuda:0")
            torch.cuda.synchronize()
        return state
    rows = other
    L, R, tokens, queries = max(keys), max(rows), sum(keys), sum(rows)
    ko, ro = _offsets(keys)[:-1, None], _offsets(rows)[:-1, None]
    la, ra = np.arange(L)[None], np.arange(R)[None]
    kn, rn = np.asarray(keys)[:, None], np.asarray(rows)[:, None]
    first, end, prefix = _ranges(case)
    state["at_key"] = _gpu(np.where(la < kn, ko + la, tokens))
    at_row = np.where(ra < rn, ro + ra, queries)
    state["at_row"] = _gpu(at_row)
    state["row_back"] = _gpu(np.concatenate([u * R + np.arange(n) for u, n in enumerate(rows)]))
    state["key_back"] = _gpu(np.concatenate([u * L + np.arange(n) for u, n in enumerate(keys)]))
    for name, x in (("first", first), ("end", end), ("prefix", prefix)):
        state[name] = _gpu(np.concatenate([x, [0]])[at_row])
    state["slopes"] = _slopes(case).float().to("cuda:0")
    if own:
        d = case["d"]
        zero = {"ln_in_g": (d,), "ln_in_b": (d,), "w1": (4 * d, d), "b1": (4 * d,), "ln_at_g": (d,), "ln_at_b": (d,), "w2": (d, d), "b2": (d,)}
        weights = {"layers": [{n: np.zeros(s, np.float32) for n, s in zero.items()} for _ in range(LAYERS)],
                   "ln_out_g": np.zeros(d, np.float32), "ln_out_b": np.zeros(d, np.float32), "w_score": np.zeros(d, np.float32), "b_score": 0.0}
        from synth.generator import ModelConfig
        state["ctx"] = rg.Context(ModelConfig(LAYERS, d, heads, case["dtype"], attention=case["form"]), weights, case["users"], 0, max(sum(rows), 8192))
        state["rows"] = rg.KvRows(handles, _offsets(rows), key_len=keys)
        state["weight_out"] = torch.empty_like(state["weight"]) if case["weigh"] else None
        state["scoring"] = rg.Scoring(
            cap=case["cap"], slopes=state["slopes"] if case["bias"] else None, window=case["window"], prefix=[case["prefix"]] * len(keys) if case["prefix"] else None,
            row_first=_gpu(first, np.int32) if case["session"] else None, row_position=state["row_pos"] if case["gaps"] else None,
            key_position=state["key_pos"] if case["gaps"] else None, token_off=_offsets(keys)[:-1])
        torch.cuda.synchronize()
    return state


def _rotate_plain(x, case, pos, freq):
    heads, dim = case["heads"], case["dim"]
    t = pos.double()[:, None] * freq[None]
    if case["transposed"]:
        t = -t
    cos, sin = (f(t).float()[:, None] * _gain(case) for f in (torch.cos, torch.sin))       # [rows, 1, dim / 2]
    y = x.float().view(x.shape[0], heads, -1).clone()
    a, b = (slice(0, dim // 2), slice(dim // 2, dim)) if case["layout"] == "half" else (slice(0, dim, 2), slice(1, dim, 2))
    u, v = y[..., a].clone(), y[..., b].clone()
    y[..., a], y[..., b] = u * cos - v * sin, u * sin + v * cos
    return y.view(x.shape).to(x.dtype)


def run(state):
    case = state["case"]
    if own:
        import paper_2601_01712_amd as rg
        if case["call"] == "rotate":
            out = rg.relaygr_rotary(state["cfg"], state["rope"], state["pos"], state["q"], state.get("k"), transposed=case["transposed"])
            return list(out) if case["both"] else [out]
        if case["call"] == "attend":
            out = rg.relaygr_cache_attend_scored(state["ctx"], state["pool"], LAYER, state["rows"], state["q"], state["scoring"], causal=case["causal"],
                                                 weight=state.get("weight"), weight_out=state["weight_out"])
            return [out, state["weight_out"]] if case["weigh"] else [out]
        rg.relaygr_kv_pool_evict(state["pool"], state["rows"], state["weight"], token_off=state["token_off"], first=case["first"], recent=case["recent"], to=state["handles"],
                                 kept=state["kept"], weight_out=state["weight_out"], position=state["pos"], position_out=state["pos_out"])
        held = [x for layer in range(LAYERS) for x in rg.relaygr_kv_pool_read(state["pool"], layer, state["read"])]
        return [state["kept"], state["weight_out"], state["pos_out"], *held]
    if case["call"] == "rotate":
        return [_rotate_plain(state[n], case, state["pos"], state["freq"]) for n in ("q", "k") if n in state]
    d, heads, dtype = case["d"], case["heads"], _TORCH[case["dtype"]]
    dh = d // heads
    if case["call"] == "evict":
        w = torch.cat([state["weight"], state["weight"].new_full((1,), -math.inf)])[state["at"]]
        w = w.masked_fill(state["must"], math.inf)
        order = torch.sort(w, dim=1, descending=True, stable=True)[1][:, :state["stay"].shape[1]]       # ties: lowest index first
        order = torch.sort(order.masked_fill(~state["stay"], w.shape[1]), dim=1)[0]
        kept = order.reshape(-1)[state["back"]]
        token = state["token0"] + kept
        out = [kept.int(), state["weight"][token], state["pos"][token]]
        blocks = sum(_blocks(m) for m in _evict_lengths(case)[1])
        for layer in range(LAYERS):
            for name in "kv":
                x = _dequantise(state[f"{name}{layer}_codes"], state[f"{name}{layer}_exp"]).view(-1, d)
                y = x.new_zeros((blocks * BLOCK, d))
                y[state["to"]] = x[state["held"][token]]
                out.append(_dequantise(*_quantise(y.view(-1, BLOCK, heads, dh))).view(-1, d)[state["to"]].to(dtype))
        return out
    k, v = (_dequantise(state[n + "_codes"], state[n + "_exp"]).view(-1, d)[state["held"]] for n in ("k", "v"))
    q = torch.cat([state["q"].float(), k.new_zeros(1, d)])[state["at_row"]].view(*state["at_row"].shape, heads, dh).transpose(1, 2).contiguous()
    k, v = (torch.cat([x, x.new_zeros(1, d)])[state["at_key"]].view(*state["at_key"].shape, heads, dh) for x in (k, v))
    s = (q @ k.permute(0, 2, 3, 1).contiguous()) / math.sqrt(dh)                                  # [users, heads, rows, keys]
    if case["cap"]:
        s = torch.tanh(s / case["cap"]) * case["cap"]
    if case["bias"]:
        pad = state["key_pos"].new_zeros(1)
        apart = (torch.cat([state["row_pos"], pad])[state["at_row"]][:, :, None] - torch.cat([state["key_pos"], pad])[state["at_key"]][:, None, :]).abs()
        s = s - state["slopes"][None, :, None, None] * apart[:, None].float()
    place = torch.arange(s.shape[-1], device=s.device)
    first, end, prefix = (state[n][:, None, :, None] for n in ("first", "end", "prefix"))                    # [users, 1, rows, 1]
    see = (place < prefix) | ((place >= first) & (place < end))
    if case["form"] == "softmax":
        s = s.masked_fill(~see, -math.inf)
        p = torch.exp(s - s.amax(dim=-1, keepdim=True).clamp(min=torch.finfo(s.dtype).min))
        p = p / p.sum(dim=-1, keepdim=True).clamp(min=1e-30)
    else:
        p = (s * torch.sigmoid(s)).masked_fill(~see, 0.0) / (prefix + end - first).clamp(min=1)
    o = (p @ v.transpose(1, 2).contiguous()).transpose(1, 2).reshape(-1, d)
    out = [o[state["row_back"]].to(dtype)]
    if case["weigh"]:
        out.append(state["weight"] + p.abs().sum(dim=(1, 2)).reshape(-1)[state["key_back"]])
    return out


def exact(case, seed):
    """From the definitions in 64 bits: an e4m3 value has four significant bits, the smallest step is 2^-9."""
    raw = _inputs(case, seed)
    heads, d = case["heads"], case["d"]
    dh = d // heads

    def two_to(e):
        return ((e.long() + 1023) << 52).view(torch.float64)

    def held(x):
        """What a cache of these tokens stands for, x [tokens, d] from a block's start on."""
        n = x.shape[0]
        y = torch.zeros((_blocks(n) * BLOCK, d), dtype=torch.float64, device=x.device)
        y[:n] = x
        y = y.view(-1, BLOCK, heads, dh)
        top = y.abs().amax(dim=(1, 3), keepdim=True).clamp(min=2.0 ** -90)
        under = two_to(torch.frexp(top)[1] - 1)             # the power of two at or under the largest value
        scale = torch.where(top > 1.75 * under, under / 128, under / 256)
        y = y / scale
        step = two_to(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
        return (torch.round(y / step) * step * scale).view(-1, d)[:n]

    if case["call"] == "rotate":
        dim, half = case["dim"], case["dim"] // 2
        out = []
        for name in ("q", "k"):
            if name not in raw:
                continue
            x = raw[name].double().view(-1, heads, dh)
            y = x.clone()
            for i in range(half):
                f = math.exp(-2.0 * i / dim * math.log(BASE))
                turns = case["original"] * f / (2 * math.pi)
                whole = min(max((turns - TURNS_LOW) / (TURNS_HIGH - TURNS_LOW), 0.0), 1.0) if case["original"] else 0.0
                angle = raw["pos"].double()[:, None] * (whole * f + (1.0 - whole) * f / case["factor"]) * (-1.0 if case["transposed"] else 1.0)
                a, b = (i, i + half) if case["layout"] == "half" else (2 * i, 2 * i + 1)
                turn = torch.polar(torch.full_like(angle, _gain(case)), angle) * torch.complex(x[..., a], x[..., b])
                y[..., a], y[..., b] = turn.real, turn.imag
            out.append(y.view(-1, d))
        return out
    if case["call"] == "evict":
        keys, keep = _evict_lengths(case)
        ko = _offsets(keys)
        weight = raw["weight"].double().cpu().numpy()
        kept, values = [], [[] for _ in range(2 * LAYERS)]
        for u, (n, m) in enumerate(zip(keys, keep)):
            w = weight[ko[u]:ko[u + 1]].copy()
            w[:case["first"]] = np.inf
            w[max(n - case["recent"], 0):] = np.inf
            mine = np.sort(np.lexsort((np.arange(n), -w))[:m])
            kept.append(mine)
            for i, name in enumerate(f"{name}{layer}" for layer in range(LAYERS) for name in "kv"):
                values[i].append(held(held(raw[name][ko[u]:ko[u + 1]].double())[_gpu(mine)]))
        token = _gpu(np.concatenate([o + mine for o, mine in zip(ko, kept)]))
        return [_gpu(np.concatenate(kept)), raw["weight"][token].double(), raw["pos"][token].long(), *[torch.cat(x) for x in values]]
    keys, rows = _lengths(case)
    ko, ro = _offsets(keys), _offsets(rows)
    first, end, prefix = (_gpu(x) for x in _ranges(case))
    slopes = _slopes(case).float().double()
    out, weights = [], []
    for u, (n, m) in enumerate(zip(keys, rows)):
        k, v = (held(raw[name][ko[u]:ko[u + 1]].double()) for name in ("k", "v"))
        r = slice(int(ro[u]), int(ro[u + 1]))
        q = raw["q"][r].double()
        j = torch.arange(n, device=q.device)[None]
        see = (j < prefix[r, None]) | ((first[r, None] <= j) & (j < end[r, None]))
        count = see.sum(dim=1, keepdim=True)
        apart = (raw["row_pos"][r].double()[:, None] - raw["key_pos"][ko[u]:ko[u + 1]].double()[None]).abs()
        of_heads, total = [], torch.zeros(n, dtype=torch.float64, device=q.device)
        for h in range(heads):
            cols = slice(h * dh, (h + 1) * dh)
            s = q[:, cols] @ k[:, cols].T.contiguous() / math.sqrt(dh)
            if case["cap"]:
                e = torch.exp(-2.0 / case["cap"] * s.abs())
                s = torch.sign(s) * case["cap"] * (1.0 - e) / (1.0 + e)
            if case["bias"]:
                s = s - float(slopes[h]) * apart
            if case["form"] == "softmax":
                w = torch.softmax(torch.where(see, s, -math.inf), dim=1)
                w = torch.where(count > 0, w, 0.0)
            else:
                w = torch.where(see, s / (1.0 + torch.exp(-s)), 0.0) / count.clamp(min=1)
            total += w.abs().sum(dim=0)
            of_heads.append(w @ v[:, cols].contiguous())
        out.append(torch.cat(of_heads, dim=1))
        weights.append(total)
    result = [torch.cat(out)]
    if case["weigh"]:
        result.append(raw["weight"].double() + torch.cat(weights))
    return result
