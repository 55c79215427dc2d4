"""The 8-bit K/V cache in 64 bits, from its definition (numpy; shares no code with the library), and what the GPU tests of it need."""
import ctypes as C
import functools
import os
import shutil
import subprocess
import tempfile

import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
import synth

BLOCK = 64
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16}
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # of a rounding to the type, relative
TOP = {"bf16": 120, "fp16": 8}                          # exponent of a block that holds the type's largest values


def e4m3(y):
    """The e4m3 number nearest to y (|y| <= 448), ties to the even mantissa; NaN stays."""
    a = np.abs(y)
    with np.errstate(invalid="ignore"):
        exp = np.frexp(np.maximum(a, 2.0 ** -6))[1] - 1     # of the binade; subnormals share 2^-6's step
        step = np.ldexp(1.0, exp - 3)
        return np.copysign(np.rint(a / step) * step, y)


def exponent(block):
    """Exponent of the scale of an array of values."""
    a = np.abs(block[np.isfinite(block)])
    top = a.max() if a.size else 0.0
    if top == 0.0:
        return -100
    m, x = np.frexp(top)                                    # top = m * 2^x
    return int(max(x - 9 + (1 if 2 * m > 1.75 else 0), -100))


def held(x, dtype):
    """What a cache of the tokens x [n, heads, dh] stands for, written from a block's start."""
    out = np.array(x, dtype=np.float64)
    for b in range(0, x.shape[0], BLOCK):
        for h in range(x.shape[1]):
            blk = out[b:b + BLOCK, h]
            e = exponent(blk)
            y = np.ldexp(np.where(np.isfinite(blk), blk, np.nan), -e)
            out[b:b + BLOCK, h] = e4m3(np.clip(y, -240.0, 240.0) if e == TOP[dtype] else y) * 2.0 ** e
    return out


class Entry:
    """One layer's K or V of one entry."""

    def __init__(self, length, heads, dh, dtype):
        self.x, self.dtype = np.zeros((length, heads, dh)), dtype

    def write(self, first, rows):
        n = rows.shape[0]
        if n == 0:
            return
        b0, end = first // BLOCK * BLOCK, first + n
        self.x[b0:end] = held(np.concatenate([self.x[b0:first], rows]), self.dtype)
        self.x[end:min(-(-end // BLOCK) * BLOCK, self.x.shape[0])] = 0.0


def attend(q, k, v, seen, form, dtype):
    """(out, bound) of rows q [m, heads, dh] over k, v [n, heads, dh], row i seeing seen[i] of them: the formula, and how far a kernel may be
    from it that rounds each weight and the output to the type and keeps everything else in 32 bits."""
    m, heads, dh = q.shape
    alpha, u = 1.0 / np.sqrt(dh), HALF_STEP[dtype]
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for h in range(heads):
        s = alpha * (q[:, h] @ k[:, h].T)
        # the score's rounding: dh products and sums and a scaling, 2^-24 each, of the sum of magnitudes
        ds = (dh + 8) * 2.0 ** -24 * alpha * (np.abs(q[:, h]) @ np.abs(k[:, h]).T)
        see = np.arange(k.shape[0])[None] < np.asarray(seen)[:, None]
        n = np.maximum(np.asarray(seen)[:, None], 1)
        if form == "softmax":
            t = np.where(see, s, -np.inf)
            w = np.where(see, np.exp(t - np.max(t, axis=1, keepdims=True, initial=-1e300)), 0.0)
            w = w / np.maximum(w.sum(axis=1, keepdims=True), 1e-300)
            worst = np.max(np.where(see, ds, 0.0), axis=1, keepdims=True, initial=0.0)
            dw = w * (u + 2 * (ds + worst) + 2.0 ** -20)       # own exponential's argument, the others' in the denominator
        else:
            w = np.where(see, s / (1.0 + np.exp(np.minimum(-s, 700.0))), 0.0) / n
            dw = np.abs(w) * (u + 2.0 ** -20) + np.where(see, 1.1 * ds, 0.0) / n      # |SiLU'| < 1.1
        if dtype == "fp16":      # weights below 2^-14 are multiples of 2^-24 (softmax: against a largest weight of at least 1)
            dw = dw + np.where(see, 2.0 ** -25, 0.0) / (1.0 if form == "softmax" else n)
        av = np.abs(v[:, h])
        out[:, h] = w @ v[:, h]
        sums = np.abs(w) @ av
        bound[:, h] = dw @ av + k.shape[0] * 2.0 ** -24 * sums + u * (np.abs(out[:, h]) + dw @ av) + 2.0 ** -25
    return out, bound


def seen_by_rows(keys, rows, causal):
    return np.maximum(keys - rows + 1 + np.arange(rows), 0) if causal else np.full(rows, keys)


def offsets(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def values(rng, n, d, dtype, spread=0.6):
    """Rows of SiLU activations whose features differ in size, in the storage type, and as float64."""
    gain = np.exp(spread * rng.standard_normal(d))
    x = rng.standard_normal((n, d)) * gain
    t = torch.from_numpy((x / (1.0 + np.exp(-x))).astype(np.float32)).to(TORCH[dtype])
    return t, t.double().numpy()


def pool_for(cfg, dtype, lens, page_tokens=64, extra=2):
    pages = sum(-(-max(n, 1) // page_tokens) for n in lens) + extra
    pool = rg.KvPool(cfg, dtype, pages * rg.relaygr_kv_pool_bytes_for_q8(cfg, page_tokens, page_tokens), page_tokens, quantized=True)
    pool.slab.fill_(0x7F)       # NaN codes and huge scales: a kernel that reads what nobody wrote is noticed
    return pool, [rg.relaygr_kv_pool_alloc(pool, 100 + u, max(n, 1)) for u, n in enumerate(lens)]


def context_for(model, users, rows):
    d = model.d_model
    shapes = {"ln_in_g": (d,), "ln_in_b": (d,), "w1": (4 * d, d), "b1": (4 * d,), "ln_at_g": (d,), "ln_at_b": (d,), "w2": (d, d), "b2": (d,)}
    weights = {"layers": [{n: np.zeros(s, np.float32) for n, s in shapes.items()} for _ in range(model.n_layers)],
               "ln_out_g": np.zeros(d, np.float32), "ln_out_b": np.zeros(d, np.float32), "w_score": np.zeros(d, np.float32), "b_score": 0.0}
    return rg.Context(model, weights, users, 0, rows)


def model(d, heads, dtype, form="silu", layers=2):
    return synth.ModelConfig(layers, d, heads, dtype, attention=form)


@functools.lru_cache(maxsize=None)
def rule_shim():
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    with tempfile.TemporaryDirectory() as tmp:
        lib = os.path.join(tmp, "attend_rule.so")
        src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "attend_rule_shim.cpp")
        subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", src, "-o", lib], check=True)
        return C.CDLL(lib)


def attend_rule(rows, keys, heads, dh, n_cus=256):
    """What a launch of attention takes: 32-row blocks of an item, whether codes are loaded once, key tiles of a piece, most pieces of a user."""
    both = [(m, n) for m, n in zip(rows, keys) if m > 0]
    r, k = (np.array(x, np.int32) for x in zip(*both))
    out = np.zeros(4, np.int32)
    rule_shim().attend_rule_of(len(both), r.ctypes.data_as(C.c_void_p), k.ctypes.data_as(C.c_void_p), heads, dh, n_cus, out.ctypes.data_as(C.c_void_p))
    return dict(zip(("blocks", "once", "piece", "parts"), out.tolist()))
