"""ctypes binding of librelaygr.so: argument marshalling only.

Every function named relaygr_* below forwards to the C entry point of the same
name (include/relaygr.h).  PyTorch supplies device memory and the current HIP
stream; no step of the path runs in Python or in PyTorch ops.  If the library
is missing it is built once with hipcc; if that fails the import fails.
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Optional, Sequence

import numpy as np
import torch

from . import build as _build

RELAYGR_OK, RELAYGR_EINVAL, RELAYGR_ENOSPC, RELAYGR_ENOENT, RELAYGR_EHIP, RELAYGR_EBUSY = 0, -1, -2, -3, -4, -5
RELAYGR_TRIGGER_NOT_AT_RISK, RELAYGR_TRIGGER_ADMIT, RELAYGR_TRIGGER_REFUSED = 0, 1, 2
RELAYGR_DTYPE_FP32, RELAYGR_DTYPE_BF16, RELAYGR_DTYPE_FP16 = 0, 1, 2
RELAYGR_NO_CACHE = 0
RELAYGR_TILE_TOKENS = 64

EXPORTS = [
    "relaygr_kv_footprint_bytes", "relaygr_kv_pool_bytes_for", "relaygr_scratch_bytes",
    "relaygr_ctx_create", "relaygr_ctx_destroy", "relaygr_ctx_set_attention",
    "relaygr_kv_pool_create", "relaygr_kv_pool_destroy", "relaygr_kv_pool_alloc", "relaygr_kv_pool_free",
    "relaygr_kv_pool_lookup", "relaygr_kv_pool_entry_len", "relaygr_kv_pool_stats", "relaygr_kv_pool_locate",
    "relaygr_prefill_prefix", "relaygr_rank_with_cache", "relaygr_rank_full_recompute",
    "relaygr_rank_with_cache_static", "relaygr_static_scratch_bytes",
    "relaygr_ctx_profile_enable", "relaygr_ctx_profile_sample", "relaygr_ctx_profile_read",
    "relaygr_kv_pool_entry_bytes", "relaygr_kv_pool_spill", "relaygr_kv_pool_reload",
    "relaygr_expander_create", "relaygr_expander_destroy", "relaygr_expander_retire",
    "relaygr_expander_alloc", "relaygr_expander_trim", "relaygr_expander_lookup", "relaygr_expander_stats",
    "relaygr_expander_set_reload_rate",
    "relaygr_admission_budget_compute", "relaygr_slot_throughput",
    "relaygr_trigger_create", "relaygr_trigger_destroy", "relaygr_trigger_admit", "relaygr_trigger_release",
    "relaygr_trigger_stats",
    "relaygr_kv_footprint_bytes_q8", "relaygr_kv_pool_bytes_for_q8", "relaygr_kv_pool_create_q8",
    "relaygr_kv_pool_write", "relaygr_kv_pool_read", "relaygr_cache_attend",
    "relaygr_rope_init", "relaygr_rotary", "relaygr_cache_attend_scored", "relaygr_kv_pool_evict",
    "relaygr_last_error",
]
EXPANDER_STATS = ["hbm_hits", "dram_hits", "misses", "refusals", "spills", "dram_evictions", "dram_bytes", "dram_entries",
                  "hbm_evictions", "hbm_reclaimable"]
KERNEL_CLASSES = ["setup", "ln", "f1", "attn", "gate", "f2", "score"]


class ModelConfigC(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_heads", C.c_int32),
                ("dtype", C.c_int32), ("ln_eps", C.c_float)]


class LayerWeightsC(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in
                ("ln_in_g", "ln_in_b", "w1", "b1", "ln_at_g", "ln_at_b", "w2", "b2")]


class WeightsC(C.Structure):
    _fields_ = [("layers", C.POINTER(LayerWeightsC)), ("ln_out_g", C.c_void_p), ("ln_out_b", C.c_void_p),
                ("w_score", C.c_void_p), ("b_score", C.c_float)]


class BatchC(C.Structure):
    _fields_ = [("n_users", C.c_int32),
                ("user_ids", C.POINTER(C.c_uint64)),
                ("handles", C.POINTER(C.c_uint64)),
                ("prefix_emb", C.c_void_p), ("prefix_off", C.POINTER(C.c_int32)),
                ("suffix_emb", C.c_void_p), ("suffix_off", C.POINTER(C.c_int32)),
                ("cand_emb", C.c_void_p), ("cand_off", C.POINTER(C.c_int32))]


class KvRowsC(C.Structure):
    _fields_ = [("n_users", C.c_int32), ("handles", C.POINTER(C.c_uint64)), ("row_off", C.POINTER(C.c_int32)),
                ("first_token", C.POINTER(C.c_int32)), ("key_len", C.POINTER(C.c_int32))]


class RopeC(C.Structure):
    _fields_ = [("dim", C.c_int32), ("layout", C.c_int32), ("gain", C.c_float), ("reserved", C.c_int32), ("turns", C.c_uint64 * 64)]


class ScoringC(C.Structure):
    _fields_ = [("cap", C.c_float), ("window", C.c_int32), ("slopes", C.c_void_p), ("prefix", C.POINTER(C.c_int32)), ("row_first", C.c_void_p),
                ("row_end", C.c_void_p), ("row_position", C.c_void_p), ("key_position", C.c_void_p), ("token_off", C.POINTER(C.c_int64))]


class KvEvictionC(C.Structure):
    _fields_ = [("first", C.c_int32), ("recent", C.c_int32), ("to", C.c_void_p), ("weight", C.c_void_p), ("position", C.c_void_p),
                ("token_off", C.c_void_p), ("kept", C.c_void_p), ("weight_out", C.c_void_p), ("position_out", C.c_void_p),
                ("out_off", C.c_void_p)]


class AdmissionParamsC(C.Structure):
    _fields_ = [("q_m", C.c_double), ("model_slots", C.c_int32), ("kv_p99_bytes", C.c_double),
                ("hbm_bytes", C.c_double), ("r1", C.c_double), ("n_instances", C.c_int32),
                ("r2", C.c_double), ("t_life_s", C.c_double)]


class AdmissionBudgetC(C.Structure):
    _fields_ = [(n, C.c_double) for n in
                ("max_live_caches", "q_admit_hbm", "q_admit_compute", "q_admit", "q_max")]


class RelayGRError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__(f"relaygr error {code}: {message}")
        self.code = code


_lib = None


def load_library() -> C.CDLL:
    """Loads librelaygr.so from the package directory (building it first if it is absent)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_build.LIB):
        _build.build()
    lib = C.CDLL(_build.LIB)
    vp, i32, i64, u64, sz = C.c_void_p, C.c_int32, C.c_int64, C.c_uint64, C.c_size_t
    P = C.POINTER
    sig = {
        "relaygr_kv_footprint_bytes": (sz, [P(ModelConfigC), i32]),
        "relaygr_kv_pool_bytes_for": (sz, [P(ModelConfigC), i32, i32]),
        "relaygr_scratch_bytes": (sz, [P(ModelConfigC), i32, i64, i64]),
        "relaygr_ctx_create": (C.c_int, [P(ModelConfigC), P(WeightsC), vp, sz, P(vp)]),
        "relaygr_ctx_destroy": (None, [vp]),
        "relaygr_kv_pool_create": (C.c_int, [P(ModelConfigC), vp, sz, i32, P(vp)]),
        "relaygr_kv_pool_destroy": (None, [vp]),
        "relaygr_kv_pool_alloc": (C.c_int, [vp, u64, i32, P(u64)]),
        "relaygr_kv_pool_free": (C.c_int, [vp, u64]),
        "relaygr_kv_pool_lookup": (C.c_int, [vp, u64, P(u64)]),
        "relaygr_kv_pool_entry_len": (C.c_int, [vp, u64, P(i32)]),
        "relaygr_kv_pool_stats": (C.c_int, [vp, P(i64), P(i64), P(i64), P(i64)]),
        "relaygr_kv_pool_locate": (C.c_int, [vp, u64, i32, i32, i32, P(i64), P(i64)]),
        "relaygr_prefill_prefix": (C.c_int, [vp, vp, P(BatchC), vp]),
        "relaygr_rank_with_cache": (C.c_int, [vp, vp, P(BatchC), vp, vp]),
        "relaygr_rank_full_recompute": (C.c_int, [vp, P(BatchC), vp, vp]),
        "relaygr_rank_with_cache_static": (C.c_int, [vp, vp, P(BatchC), vp, vp]),
        "relaygr_static_scratch_bytes": (sz, []),
        "relaygr_ctx_profile_enable": (C.c_int, [vp, C.c_uint32]),
        "relaygr_ctx_profile_sample": (C.c_int, [vp, i32]),
        "relaygr_ctx_set_attention": (C.c_int, [vp, i32]),
        "relaygr_ctx_profile_read": (C.c_int, [vp, i32, P(C.c_double), P(i64)]),
        "relaygr_kv_pool_entry_bytes": (sz, [vp, u64]),
        "relaygr_kv_pool_spill": (C.c_int, [vp, u64, vp, sz, vp]),
        "relaygr_kv_pool_reload": (C.c_int, [vp, u64, i32, vp, sz, vp, P(u64)]),
        "relaygr_expander_create": (C.c_int, [vp, sz, i32, P(vp)]),
        "relaygr_expander_destroy": (None, [vp]),
        "relaygr_expander_retire": (C.c_int, [vp, u64, vp]),
        "relaygr_expander_alloc": (C.c_int, [vp, u64, i32, P(u64)]),
        "relaygr_expander_trim": (C.c_int, [vp, i32]),
        "relaygr_expander_set_reload_rate": (C.c_int, [vp, C.c_double, C.c_double]),
        "relaygr_expander_lookup": (C.c_int, [vp, u64, vp, P(u64), P(i32)]),
        "relaygr_expander_stats": (C.c_int, [vp, P(i64)]),
        "relaygr_admission_budget_compute": (C.c_int, [P(AdmissionParamsC), P(AdmissionBudgetC)]),
        "relaygr_slot_throughput": (C.c_double, [C.c_double]),
        "relaygr_trigger_create": (C.c_int, [P(AdmissionBudgetC), i32, P(vp)]),
        "relaygr_trigger_destroy": (None, [vp]),
        "relaygr_trigger_admit": (C.c_int, [vp, C.c_double, i32]),
        "relaygr_trigger_release": (C.c_int, [vp]),
        "relaygr_trigger_stats": (C.c_int, [vp, P(i64), P(i64), P(i64), P(i64)]),
        "relaygr_kv_footprint_bytes_q8": (sz, [P(ModelConfigC), i32]),
        "relaygr_kv_pool_bytes_for_q8": (sz, [P(ModelConfigC), i32, i32]),
        "relaygr_kv_pool_create_q8": (C.c_int, [P(ModelConfigC), vp, sz, i32, P(vp)]),
        "relaygr_kv_pool_write": (C.c_int, [vp, i32, P(KvRowsC), vp, i64, vp, i64, vp]),
        "relaygr_kv_pool_read": (C.c_int, [vp, i32, P(KvRowsC), vp, i64, vp, i64, vp]),
        "relaygr_cache_attend": (C.c_int, [vp, vp, i32, P(KvRowsC), i32, vp, i64, vp, i64, vp]),
        "relaygr_rope_init": (C.c_int, [P(RopeC), i32, i32, C.c_double, C.c_double, i32, C.c_double, C.c_double, C.c_float]),
        "relaygr_rotary": (C.c_int, [P(ModelConfigC), P(RopeC), i32, vp, i32, vp, i64, vp, i64, vp, i64, vp, i64, vp]),
        "relaygr_cache_attend_scored": (C.c_int, [vp, vp, i32, P(KvRowsC), i32, P(ScoringC), vp, i64, vp, i64, vp, vp, vp]),
        "relaygr_kv_pool_evict": (C.c_int, [vp, P(KvRowsC), P(KvEvictionC), vp]),
        "relaygr_last_error": (C.c_char_p, []),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)   # AttributeError here means the library lacks a declared symbol
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _check(rc: int) -> None:
    if rc != RELAYGR_OK:
        raise RelayGRError(rc, load_library().relaygr_last_error().decode("utf-8", "replace"))


def relaygr_last_error() -> str:
    return load_library().relaygr_last_error().decode("utf-8", "replace")


def _dtype_code(dtype: str) -> int:
    return {"fp32": RELAYGR_DTYPE_FP32, "bf16": RELAYGR_DTYPE_BF16, "fp16": RELAYGR_DTYPE_FP16}[dtype]


_TORCH_DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _torch_dtype(dtype: str):
    return _TORCH_DTYPES[dtype]


def make_config(n_layers: int, d_model: int, n_heads: int, dtype: str, ln_eps: float = 1e-5) -> ModelConfigC:
    return ModelConfigC(n_layers, d_model, n_heads, _dtype_code(dtype), ln_eps)


def relaygr_kv_footprint_bytes(cfg: ModelConfigC, prefix_len: int) -> int:
    return load_library().relaygr_kv_footprint_bytes(C.byref(cfg), prefix_len)


def relaygr_kv_pool_bytes_for(cfg: ModelConfigC, prefix_len: int, page_tokens: int) -> int:
    return load_library().relaygr_kv_pool_bytes_for(C.byref(cfg), prefix_len, page_tokens)


def relaygr_scratch_bytes(cfg: ModelConfigC, max_users: int, max_prefix_tokens: int, max_new_tokens: int) -> int:
    return load_library().relaygr_scratch_bytes(C.byref(cfg), max_users, max_prefix_tokens, max_new_tokens)


def _stream_ptr(stream) -> int:
    """HIP stream handle of a torch stream (default: torch's current stream) or a raw hipStream_t given as an int."""
    if isinstance(stream, int):
        return stream
    s = stream if stream is not None else torch.cuda.current_stream()
    return int(s.cuda_stream)


class Context:
    """relaygr_ctx plus the device tensors it references (weights, scratch)."""

    def __init__(self, model_cfg, weights: dict, max_users: int, max_prefix_tokens: int, max_new_tokens: int,
                 device: str = "cuda:0"):
        lib = load_library()
        self.dtype = model_cfg.dtype
        self.cfg = make_config(model_cfg.n_layers, model_cfg.d_model, model_cfg.n_heads, model_cfg.dtype, model_cfg.ln_eps)
        td = _torch_dtype(self.dtype)
        self.device = torch.device(device)
        self._keep = []

        def dev(a):
            t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(self.device).to(td).contiguous()
            self._keep.append(t)
            return t.data_ptr()

        layers = (LayerWeightsC * model_cfg.n_layers)()
        for l, lw in enumerate(weights["layers"]):
            for name, _ in LayerWeightsC._fields_:
                setattr(layers[l], name, dev(lw[name]))
        self._layers = layers
        wc = WeightsC(layers, dev(weights["ln_out_g"]), dev(weights["ln_out_b"]), dev(weights["w_score"]),
                      float(weights["b_score"]))
        nbytes = relaygr_scratch_bytes(self.cfg, max_users, max_prefix_tokens, max_new_tokens)
        if nbytes == 0:
            raise RelayGRError(RELAYGR_EINVAL, "relaygr_scratch_bytes rejected the configuration")
        self.scratch = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.scratch_bytes = nbytes
        h = C.c_void_p()
        _check(lib.relaygr_ctx_create(C.byref(self.cfg), C.byref(wc), self.scratch.data_ptr(), nbytes, C.byref(h)))
        self.handle = h
        form = getattr(model_cfg, "attention", "silu")
        if form != "silu":
            relaygr_ctx_set_attention(self, form)

    def close(self):
        if getattr(self, "handle", None):
            torch.cuda.synchronize(self.device)
            load_library().relaygr_ctx_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


ATTENTION_FORMS = {"silu": 0, "softmax": 1}


def relaygr_ctx_set_attention(ctx: Context, form: str) -> None:
    """Selects the context's attention form: "silu" (pointwise SiLU, the default) or "softmax"."""
    if form not in ATTENTION_FORMS:
        raise RelayGRError(RELAYGR_EINVAL, f"unknown attention form {form!r}")
    _check(load_library().relaygr_ctx_set_attention(ctx.handle, ATTENTION_FORMS[form]))


def relaygr_ctx_profile_enable(ctx: Context, classes: Sequence[str]) -> None:
    mask = 0
    for c in classes:
        mask |= 1 << KERNEL_CLASSES.index(c)
    _check(load_library().relaygr_ctx_profile_enable(ctx.handle, mask))


def relaygr_ctx_profile_sample(ctx: Context, every_n_calls: int) -> None:
    _check(load_library().relaygr_ctx_profile_sample(ctx.handle, every_n_calls))


def relaygr_ctx_profile_read(ctx: Context, kernel_class: str):
    """(total milliseconds, launches) of one kernel class since profiling was enabled."""
    ms, n = C.c_double(), C.c_int64()
    _check(load_library().relaygr_ctx_profile_read(ctx.handle, KERNEL_CLASSES.index(kernel_class), C.byref(ms), C.byref(n)))
    return ms.value, n.value


class KvPool:
    """relaygr_kv_pool over a torch-allocated device slab; quantized: K and V in 8 bits (relaygr_kv_pool_create_q8)."""

    def __init__(self, cfg: ModelConfigC, dtype: str, slab_bytes: int, page_tokens: int = 256, device: str = "cuda:0",
                 quantized: bool = False):
        lib = load_library()
        self.cfg = cfg
        self.dtype = dtype
        self.quantized = quantized
        self.device = torch.device(device)
        self.slab = torch.empty(slab_bytes, dtype=torch.uint8, device=self.device)
        h = C.c_void_p()
        create = lib.relaygr_kv_pool_create_q8 if quantized else lib.relaygr_kv_pool_create
        _check(create(C.byref(cfg), self.slab.data_ptr(), slab_bytes, page_tokens, C.byref(h)))
        self.handle = h

    def elements(self) -> torch.Tensor:
        """The slab viewed in the storage dtype, or as its 8-bit codes (for inspection with relaygr_kv_pool_locate)."""
        return self.slab.view(torch.float8_e4m3fn if self.quantized else _torch_dtype(self.dtype))

    def close(self):
        if getattr(self, "handle", None):
            load_library().relaygr_kv_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def relaygr_kv_pool_alloc(pool: KvPool, user_id: int, prefix_len: int) -> int:
    out = C.c_uint64(0)
    _check(load_library().relaygr_kv_pool_alloc(pool.handle, user_id, prefix_len, C.byref(out)))
    return out.value


def relaygr_kv_pool_free(pool: KvPool, handle: int) -> None:
    _check(load_library().relaygr_kv_pool_free(pool.handle, handle))


def relaygr_kv_pool_lookup(pool: KvPool, user_id: int) -> int:
    """Handle of the user's live entry, or RELAYGR_NO_CACHE if there is none."""
    out = C.c_uint64(0)
    rc = load_library().relaygr_kv_pool_lookup(pool.handle, user_id, C.byref(out))
    if rc == RELAYGR_ENOENT:
        return RELAYGR_NO_CACHE
    _check(rc)
    return out.value


def relaygr_kv_pool_entry_len(pool: KvPool, handle: int) -> int:
    out = C.c_int32(0)
    _check(load_library().relaygr_kv_pool_entry_len(pool.handle, handle, C.byref(out)))
    return out.value


def relaygr_kv_pool_stats(pool: KvPool) -> dict:
    a, b, c, d = C.c_int64(), C.c_int64(), C.c_int64(), C.c_int64()
    _check(load_library().relaygr_kv_pool_stats(pool.handle, C.byref(a), C.byref(b), C.byref(c), C.byref(d)))
    return {"pages_total": a.value, "pages_free": b.value, "live_entries": c.value, "largest_free_extent": d.value}


def relaygr_kv_pool_locate(pool: KvPool, handle: int, layer: int, token: int, feature: int):
    k, v = C.c_int64(), C.c_int64()
    _check(load_library().relaygr_kv_pool_locate(pool.handle, handle, layer, token, feature, C.byref(k), C.byref(v)))
    return k.value, v.value


# ---- 8-bit pools -----------------------------------------------------------------------------
def relaygr_kv_footprint_bytes_q8(cfg: ModelConfigC, prefix_len: int) -> int:
    return load_library().relaygr_kv_footprint_bytes_q8(C.byref(cfg), prefix_len)


def relaygr_kv_pool_bytes_for_q8(cfg: ModelConfigC, prefix_len: int, page_tokens: int) -> int:
    return load_library().relaygr_kv_pool_bytes_for_q8(C.byref(cfg), prefix_len, page_tokens)


class KvRows:
    """The host arrays of a relaygr_kv_rows: which rows of a call's tensors belong to which entry, and where in it they are.

    row_off: n_users + 1 offsets.  first_token (write, read): token of the entry that a user's first row is; None: 0.  key_len
    (attend): tokens of the entry that take part; None: all.  Made once, used in any number of calls, between which handles, first_token and
    key_len may be changed in place; row_off, which the checks of the calls' tensors go by, and which array is which are fixed."""

    def __init__(self, handles: Sequence[int], row_off: Sequence[int], first_token: Optional[Sequence[int]] = None,
                 key_len: Optional[Sequence[int]] = None):
        self.handles = np.array(handles, dtype=np.uint64)
        self.row_off = np.array(row_off, dtype=np.int32)
        self.first_token = None if first_token is None else np.array(first_token, dtype=np.int32)
        self.key_len = None if key_len is None else np.array(key_len, dtype=np.int32)
        self.n_users = self.handles.size
        for name, a, n in (("handles", self.handles, self.n_users), ("row_off", self.row_off, self.n_users + 1),
                           ("first_token", self.first_token, self.n_users), ("key_len", self.key_len, self.n_users)):
            if a is not None and a.shape != (n,):
                raise RelayGRError(RELAYGR_EINVAL, f"KvRows: {name} has shape {a.shape}, ({n},) is needed")
        self.n_rows = int(self.row_off[-1])
        self.row_off.flags.writeable = False

        def ptr(a):
            return None if a is None else a.ctypes.data_as(C.POINTER(C.c_int32))
        self.c = KvRowsC(self.n_users, self.handles.ctypes.data_as(C.POINTER(C.c_uint64)), ptr(self.row_off), ptr(self.first_token),
                         ptr(self.key_len))
        self.ref = C.byref(self.c)

    def __setattr__(self, name, value):
        if "ref" in self.__dict__ and value is not self.__dict__.get(name):     # (made: the library has the arrays' addresses; a += puts the same one back)
            raise AttributeError(f"KvRows: {name} cannot be replaced; change handles, first_token and key_len in place, or make another")
        object.__setattr__(self, name, value)


def _kv_rows_array(what: str, pool: KvPool, rows: KvRows, t: torch.Tensor):
    """(address, elements between rows) of a tensor [rows, d_model] or [rows, heads, d_head] on the pool's device."""
    d, n, shape, stride = pool.cfg.d_model, rows.n_rows, t.shape, t.stride()
    if len(shape) == 2:
        ok = shape[0] == n and shape[1] == d and (n == 0 or stride[1] == 1)     # (the strides of nothing mean nothing)
    else:
        heads = pool.cfg.n_heads
        ok = len(shape) == 3 and tuple(shape) == (n, heads, d // heads) and (n == 0 or (stride[2] == 1 and (heads == 1 or stride[1] == d // heads)))
    if not ok or t.dtype != _torch_dtype(pool.dtype) or t.device != pool.slab.device:
        raise RelayGRError(RELAYGR_EINVAL, f"{what}: needs {n} rows of {d} adjacent {pool.dtype} elements on {pool.slab.device}, got "
                                           f"{tuple(shape)} of {t.dtype} on {t.device} with strides {stride}")
    # (the stride of a single row means nothing: torch may report any)
    return (t.data_ptr() if n else None), (stride[0] if n > 1 else d)


def _kv_guard(pool: KvPool, stream):
    """What a call has to be made under to be the default one, of the current stream of the pool's device, which is also where its results are
    allocated; None if it is that already (torch's guards take several microseconds)."""
    device = pool.slab.device
    if stream is not None:
        s = torch.cuda.ExternalStream(stream, device=device) if isinstance(stream, int) else stream
        if s.device != device:
            raise RelayGRError(RELAYGR_EINVAL, f"a stream of {s.device} for a pool on {device}")
        return torch.cuda.stream(s)
    return None if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _result_rows(what: str, pool: KvPool, rows: KvRows, t: Optional[torch.Tensor]):
    """A result's tensor (made here if the caller gives none), its address and the elements between its rows."""
    if t is not None:
        return (t, *_kv_rows_array(what, pool, rows, t))
    d = pool.cfg.d_model
    t = torch.empty_strided((rows.n_rows, d), (d, 1), dtype=_torch_dtype(pool.dtype), device=pool.slab.device)     # (a microsecond less than torch.empty)
    return t, (t.data_ptr() if rows.n_rows else None), d


def relaygr_kv_pool_write(pool: KvPool, layer: int, rows: KvRows, k: torch.Tensor, v: torch.Tensor, stream=None) -> None:
    """Quantises rows of K and V ([rows, d_model] or [rows, heads, d_head]) into the entries' tokens first_token on."""
    guard = _kv_guard(pool, stream)
    if guard is not None:
        with guard:
            return relaygr_kv_pool_write(pool, layer, rows, k, v)
    kp, ks = _kv_rows_array("kv_pool_write: k", pool, rows, k)
    vp, vs = _kv_rows_array("kv_pool_write: v", pool, rows, v)
    _check(load_library().relaygr_kv_pool_write(pool.handle, layer, rows.ref, kp, ks, vp, vs, torch._C._cuda_getCurrentRawStream(pool.slab.device.index)))


def relaygr_kv_pool_read(pool: KvPool, layer: int, rows: KvRows, k: Optional[torch.Tensor] = None, v: Optional[torch.Tensor] = None,
                         stream=None):
    """(k, v): the values that tokens of the entries stand for, [rows, d_model] each (made here if not given)."""
    guard = _kv_guard(pool, stream)
    if guard is not None:
        with guard:
            return relaygr_kv_pool_read(pool, layer, rows, k, v)
    k, kp, ks = _result_rows("kv_pool_read: k", pool, rows, k)
    v, vp, vs = _result_rows("kv_pool_read: v", pool, rows, v)
    _check(load_library().relaygr_kv_pool_read(pool.handle, layer, rows.ref, kp, ks, vp, vs, torch._C._cuda_getCurrentRawStream(pool.slab.device.index)))
    return k, v


def relaygr_cache_attend(ctx: Context, pool: KvPool, layer: int, rows: KvRows, q: torch.Tensor, causal: bool = False,
                         out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One layer's attention of query rows over entries of an 8-bit pool, in the context's form: [rows, d_model] (made here if not given)."""
    if ctx.scratch.device != pool.slab.device:
        raise RelayGRError(RELAYGR_EINVAL, f"cache_attend: a context on {ctx.scratch.device} for a pool on {pool.slab.device}")
    guard = _kv_guard(pool, stream)
    if guard is not None:
        with guard:
            return relaygr_cache_attend(ctx, pool, layer, rows, q, causal, out)
    qp, qs = _kv_rows_array("cache_attend: q", pool, rows, q)
    out, op, os_ = _result_rows("cache_attend: out", pool, rows, out)
    _check(load_library().relaygr_cache_attend(ctx.handle, pool.handle, layer, rows.ref, int(causal), qp, qs, op, os_,
                                               torch._C._cuda_getCurrentRawStream(pool.slab.device.index)))
    return out


# ---- positions, scores, masks and eviction ------------------------------------------------------
ROPE_LAYOUTS = {"half": 0, "interleaved": 1}


class Rope:
    """relaygr_rope: the frequencies of rotary positions.  layout: "half" or "interleaved" pairs; factor, original_len, low, high: how positions are
    stretched (include/relaygr.h); gain: what turned features are multiplied with."""

    def __init__(self, dim: int, base: float = 10000.0, layout: str = "half", factor: float = 1.0, original_len: int = 0, low: float = 1.0,
                 high: float = 32.0, gain: float = 1.0):
        if layout not in ROPE_LAYOUTS:
            raise RelayGRError(RELAYGR_EINVAL, f"unknown layout {layout!r}")
        self.c = RopeC()
        _check(load_library().relaygr_rope_init(C.byref(self.c), dim, ROPE_LAYOUTS[layout], base, factor, original_len, low, high, gain))
        self.ref = C.byref(self.c)


def _device_guard(device: torch.device, stream):
    """What a call on tensors of a device has to be made under to be the default one, of that device's current stream; None if it is that already."""
    if stream is not None:
        s = torch.cuda.ExternalStream(stream, device=device) if isinstance(stream, int) else stream
        if s.device != device:
            raise RelayGRError(RELAYGR_EINVAL, f"a stream of {s.device} for tensors on {device}")
        return torch.cuda.stream(s)
    return None if torch.cuda.current_device() == device.index else torch.cuda.device(device)


def _vector(what: str, t: Optional[torch.Tensor], dtype, device, n: Optional[int] = None):
    """Address of a vector on the device, of n elements if n is given; None for none."""
    if t is None:
        return None
    if t.dim() != 1 or t.dtype != dtype or t.device != device or (t.numel() > 1 and t.stride(0) != 1) or (n is not None and t.numel() != n):
        raise RelayGRError(RELAYGR_EINVAL, f"{what}: needs {'' if n is None else n} adjacent {dtype} elements on {device}, got {tuple(t.shape)} of {t.dtype} on "
                                           f"{t.device} with strides {t.stride()}")
    return t.data_ptr() if t.numel() else None


def _rotary_rows(what: str, cfg: ModelConfigC, n: int, device, t: torch.Tensor):
    """(address, elements between rows) of a tensor [rows, d_model] or [rows, heads, d_head]."""
    d, heads, shape, stride = cfg.d_model, cfg.n_heads, tuple(t.shape), t.stride()
    ok = shape == (n, d) and (n == 0 or stride[1] == 1) or shape == (n, heads, d // heads) and (n == 0 or (stride[2] == 1 and (heads == 1 or stride[1] == d // heads)))
    if not ok or t.dtype != _DTYPES_BY_CODE[cfg.dtype] or t.device != device:
        raise RelayGRError(RELAYGR_EINVAL, f"{what}: needs {n} rows of {d} adjacent {_DTYPES_BY_CODE[cfg.dtype]} elements on {device}, got {shape} of {t.dtype} on "
                                           f"{t.device} with strides {stride}")
    return (t.data_ptr() if n else None), (stride[0] if n > 1 else d)


def _rotary_result(what: str, cfg: ModelConfigC, n: int, device, x: torch.Tensor, t: Optional[torch.Tensor]):
    """A result's tensor (like x, which has been checked, if the caller gives none), its address and the elements between its rows."""
    if t is not None:
        return (t, *_rotary_rows(what, cfg, n, device, t))
    t = torch.empty_like(x, memory_format=torch.contiguous_format)
    return t, (t.data_ptr() if n else None), cfg.d_model


_DTYPES_BY_CODE = {RELAYGR_DTYPE_FP32: torch.float32, RELAYGR_DTYPE_BF16: torch.bfloat16, RELAYGR_DTYPE_FP16: torch.float16}


def relaygr_rotary(cfg: ModelConfigC, rope: Rope, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None, transposed: bool = False,
                   q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream=None):
    """Rows of q (and of k) turned by their positions (int32 [rows]): q, or (q, k), made here if q_out and k_out are not given; q_out may be q, k_out k.
    transposed: by the opposite angle, which is the gradient's."""
    device = q.device
    if device.type != "cuda":
        raise RelayGRError(RELAYGR_EINVAL, f"rotary: q is on {device}")
    if k is None and k_out is not None:
        raise RelayGRError(RELAYGR_EINVAL, "rotary: k_out without k")
    guard = _device_guard(device, stream)
    if guard is not None:
        with guard:
            return relaygr_rotary(cfg, rope, positions, q, k, transposed, q_out, k_out)
    n = q.shape[0]
    pos = _vector("rotary: positions", positions, torch.int32, device, n)
    qp, qs = _rotary_rows("rotary: q", cfg, n, device, q)
    q_out, qo, qos = _rotary_result("rotary: q_out", cfg, n, device, q, q_out)
    kp = ko = None
    ks = kos = 0
    if k is not None:
        kp, ks = _rotary_rows("rotary: k", cfg, n, device, k)
        k_out, ko, kos = _rotary_result("rotary: k_out", cfg, n, device, k, k_out)
    _check(load_library().relaygr_rotary(C.byref(cfg), rope.ref, n, pos, int(transposed), qp, qs, qo, qos, kp, ks, ko, kos,
                                         torch._C._cuda_getCurrentRawStream(device.index)))
    return q_out if k is None else (q_out, k_out)


def _int32(what: str, x) -> int:
    """x, unless the struct's 32 bits would hold another number."""
    if not -2 ** 31 <= x < 2 ** 31:
        raise RelayGRError(RELAYGR_EINVAL, f"{what}: {x} is beyond 32 bits")
    return x


def _host_vector(what: str, x, dtype, n: Optional[int] = None):
    a = np.array(x, dtype=dtype)
    if a.ndim != 1 or (n is not None and a.size != n):
        raise RelayGRError(RELAYGR_EINVAL, f"{what}: has shape {a.shape}" + ("" if n is None else f", ({n},) is needed"))
    return a


class Scoring:
    """relaygr_scoring: scores and masks of relaygr_cache_attend_scored (include/relaygr.h has the formulas).

    Device tensors: slopes fp32 [heads]; row_first, row_end, row_position int32 [rows]; key_position int32, user u's token j at token_off[u] + j.
    Host: cap, window, prefix [users], token_off [users].  Made once, used in any number of calls of batches of these sizes; the tensors' contents, prefix and token_off may
    change between them in place."""

    def __init__(self, cap: float = 0.0, slopes: Optional[torch.Tensor] = None, window: int = 0, prefix: Optional[Sequence[int]] = None,
                 row_first: Optional[torch.Tensor] = None, row_end: Optional[torch.Tensor] = None, row_position: Optional[torch.Tensor] = None,
                 key_position: Optional[torch.Tensor] = None, token_off: Optional[Sequence[int]] = None):
        self.slopes, self.row_first, self.row_end, self.row_position, self.key_position = slopes, row_first, row_end, row_position, key_position
        if prefix is not None and np.size(prefix):     # (numpy would keep the low 32 bits of an array's wider elements)
            _int32("Scoring: prefix", np.min(prefix))
            _int32("Scoring: prefix", np.max(prefix))
        self.prefix = None if prefix is None else _host_vector("Scoring: prefix", prefix, np.int32)
        self.token_off = None if token_off is None else _host_vector("Scoring: token_off", token_off, np.int64)
        if key_position is not None and token_off is None:
            raise RelayGRError(RELAYGR_EINVAL, "Scoring: key_position without token_off")
        self.tensors = [x for x in (("slopes", slopes, torch.float32), ("row_first", row_first, torch.int32), ("row_end", row_end, torch.int32),
                                    ("row_position", row_position, torch.int32), ("key_position", key_position, torch.int32)) if x[1] is not None]
        self.arrays = [x for x in (("prefix", self.prefix), ("token_off", self.token_off)) if x[1] is not None]
        self.c = ScoringC(cap, _int32("Scoring: window", window), None, None if self.prefix is None else self.prefix.ctypes.data_as(C.POINTER(C.c_int32)), None, None, None, None,
                          None if self.token_off is None else self.token_off.ctypes.data_as(C.POINTER(C.c_int64)))
        if cap != 0 and self.c.cap == 0:     # (0 would be no cap at all)
            raise RelayGRError(RELAYGR_EINVAL, f"Scoring: a cap of {cap} is below what fp32 holds")
        self.ref = C.byref(self.c)

    def __setattr__(self, name, value):
        if "ref" in self.__dict__ and value is not self.__dict__.get(name):     # (made: the struct has its values)
            raise AttributeError(f"Scoring: {name} cannot be replaced; change arrays in place, or make another")
        object.__setattr__(self, name, value)

    def bind(self, pool: KvPool, rows: KvRows) -> None:
        """Checks the arrays against a batch and puts the tensors' addresses into the struct."""
        device = pool.slab.device
        for name, t, dtype in self.tensors:
            n = pool.cfg.n_heads if name == "slopes" else None if name == "key_position" else rows.n_rows
            setattr(self.c, name, _vector("Scoring: " + name, t, dtype, device, n))
        for name, a in self.arrays:
            if a.size != rows.n_users:
                raise RelayGRError(RELAYGR_EINVAL, f"Scoring: {name} of {a.size} users for a batch of {rows.n_users}")


def _tokens_fit(what: str, rows: KvRows, lens, token_off: np.ndarray, tensors) -> None:
    """Refuses tensors, by name, of which one does not hold the tokens of every user."""
    need = max((token_off + lens).tolist()) if rows.n_users else 0
    for name, t in tensors:
        if t is not None and need > t.numel():
            raise RelayGRError(RELAYGR_EINVAL, f"{what}: {name} of {t.numel()} elements does not hold every user's tokens")


def _lens(pool: KvPool, rows: KvRows):
    return rows.key_len if rows.key_len is not None else np.array([relaygr_kv_pool_entry_len(pool, int(h)) for h in rows.handles], dtype=np.int32)


def relaygr_cache_attend_scored(ctx: Context, pool: KvPool, layer: int, rows: KvRows, q: torch.Tensor, scoring: Scoring, causal: bool = False,
                                out: Optional[torch.Tensor] = None, weight: Optional[torch.Tensor] = None, weight_out: Optional[torch.Tensor] = None,
                                stream=None) -> torch.Tensor:
    """relaygr_cache_attend with scores and masks of `scoring`: [rows, d_model] (made here if not given).  weight_out (fp32, user u's token j at
    scoring.token_off[u] + j): weight, or 0 without one, plus what each token received from these rows; weight alone is added to in place."""
    if ctx.scratch.device != pool.slab.device:
        raise RelayGRError(RELAYGR_EINVAL, f"cache_attend_scored: a context on {ctx.scratch.device} for a pool on {pool.slab.device}")
    guard = _kv_guard(pool, stream)
    if guard is not None:
        with guard:
            return relaygr_cache_attend_scored(ctx, pool, layer, rows, q, scoring, causal, out, weight, weight_out)
    qp, qs = _kv_rows_array("cache_attend_scored: q", pool, rows, q)
    scoring.bind(pool, rows)
    weight_out = weight if weight_out is None else weight_out
    wi = _vector("cache_attend_scored: weight", weight, torch.float32, pool.slab.device)
    wo = _vector("cache_attend_scored: weight_out", weight_out, torch.float32, pool.slab.device)
    if scoring.token_off is not None and (weight_out is not None or scoring.key_position is not None):
        _tokens_fit("cache_attend_scored", rows, _lens(pool, rows), scoring.token_off,
                    (("key_position", scoring.key_position), ("weight", weight), ("weight_out", weight_out)))
    out, op, os_ = _result_rows("cache_attend_scored: out", pool, rows, out)
    _check(load_library().relaygr_cache_attend_scored(ctx.handle, pool.handle, layer, rows.ref, int(causal), scoring.ref, qp, qs, op, os_, wi, wo,
                                                      torch._C._cuda_getCurrentRawStream(pool.slab.device.index)))
    return out


def relaygr_kv_pool_evict(pool: KvPool, rows: KvRows, weight: torch.Tensor, token_off: Sequence[int], first: int = 0, recent: int = 0,
                          to: Optional[Sequence[int]] = None, kept: Optional[torch.Tensor] = None, weight_out: Optional[torch.Tensor] = None,
                          position: Optional[torch.Tensor] = None, position_out: Optional[torch.Tensor] = None, out_off: Optional[Sequence[int]] = None,
                          stream=None) -> torch.Tensor:
    """Evicts the tokens with the least weight: rows.row_off says how many of the first rows.key_len tokens of each entry stay.  Returns `kept` (int32
    [rows.n_rows], made here if not given): the places of those that stay.  Where weight_out is weight, the places behind them still hold weights of
    before: clear them before tokens that are written there have theirs added up."""
    guard = _kv_guard(pool, stream)
    if guard is not None:
        with guard:
            return relaygr_kv_pool_evict(pool, rows, weight, token_off, first, recent, to, kept, weight_out, position, position_out, out_off)
    device, n = pool.slab.device, rows.n_users
    token_off = _host_vector("kv_pool_evict: token_off", token_off, np.int64, n)
    out_off = None if out_off is None else _host_vector("kv_pool_evict: out_off", out_off, np.int64, n)
    to = None if to is None else _host_vector("kv_pool_evict: to", to, np.uint64, n)
    kept = torch.empty(rows.n_rows, dtype=torch.int32, device=device) if kept is None else kept
    e = KvEvictionC(_int32("kv_pool_evict: first", first), _int32("kv_pool_evict: recent", recent), None if to is None else to.ctypes.data,
                    _vector("kv_pool_evict: weight", weight, torch.float32, device),
                    _vector("kv_pool_evict: position", position, torch.int32, device), token_off.ctypes.data,
                    _vector("kv_pool_evict: kept", kept, torch.int32, device, rows.n_rows), _vector("kv_pool_evict: weight_out", weight_out, torch.float32, device),
                    _vector("kv_pool_evict: position_out", position_out, torch.int32, device),
                    None if out_off is None else out_off.ctypes.data)
    _tokens_fit("kv_pool_evict", rows, _lens(pool, rows), token_off, (("weight", weight), ("position", position)))
    if weight_out is not None or position_out is not None:
        starts = rows.row_off[:-1]
        _tokens_fit("kv_pool_evict", rows, rows.row_off[1:] - starts, starts if out_off is None else out_off, (("weight_out", weight_out), ("position_out", position_out)))
    _check(load_library().relaygr_kv_pool_evict(pool.handle, rows.ref, C.byref(e), torch._C._cuda_getCurrentRawStream(device.index)))
    return kept


# ---- DRAM tier -------------------------------------------------------------------------------
def relaygr_kv_pool_entry_bytes(pool: KvPool, handle: int) -> int:
    return load_library().relaygr_kv_pool_entry_bytes(pool.handle, handle)


def relaygr_kv_pool_spill(pool: KvPool, handle: int, host: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Enqueues the copy of the entry's extent into a pinned uint8 host tensor (made here if not given)."""
    n = relaygr_kv_pool_entry_bytes(pool, handle)
    if host is None:
        host = torch.empty(n, dtype=torch.uint8, pin_memory=True)
    _check(load_library().relaygr_kv_pool_spill(pool.handle, handle, host.data_ptr(), host.numel(), _stream_ptr(stream)))
    return host


def relaygr_kv_pool_reload(pool: KvPool, user_id: int, prefix_len: int, host: torch.Tensor, stream=None) -> int:
    out = C.c_uint64(0)
    _check(load_library().relaygr_kv_pool_reload(pool.handle, user_id, prefix_len, host.data_ptr(), host.numel(),
                                                 _stream_ptr(stream), C.byref(out)))
    return out.value


class Expander:
    """relaygr_expander over a KvPool."""

    def __init__(self, pool: KvPool, dram_budget_bytes: int, max_inflight_reloads: int = 4):
        self.pool = pool
        h = C.c_void_p()
        _check(load_library().relaygr_expander_create(pool.handle, dram_budget_bytes, max_inflight_reloads, C.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            load_library().relaygr_expander_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def relaygr_expander_retire(ex: Expander, handle: int, stream=None) -> None:
    _check(load_library().relaygr_expander_retire(ex.handle, handle, _stream_ptr(stream)))


def relaygr_expander_alloc(ex: Expander, user_id: int, prefix_len: int) -> int:
    out = C.c_uint64(0)
    _check(load_library().relaygr_expander_alloc(ex.handle, user_id, prefix_len, C.byref(out)))
    return out.value


def relaygr_expander_set_reload_rate(ex: Expander, bytes_per_second: float, burst_bytes: float) -> None:
    _check(load_library().relaygr_expander_set_reload_rate(ex.handle, C.c_double(bytes_per_second), C.c_double(burst_bytes)))


def relaygr_expander_trim(ex: Expander, keep: int = 0) -> None:
    _check(load_library().relaygr_expander_trim(ex.handle, keep))


def relaygr_expander_lookup(ex: Expander, user_id: int, stream=None):
    """(handle, source) with source 0 = HBM, 1 = reloaded from DRAM; raises RelayGRError with code
    RELAYGR_ENOENT (in neither tier) or RELAYGR_EBUSY (reload limit reached)."""
    out, src = C.c_uint64(0), C.c_int32(-1)
    _check(load_library().relaygr_expander_lookup(ex.handle, user_id, _stream_ptr(stream), C.byref(out), C.byref(src)))
    return out.value, src.value


def relaygr_expander_stats(ex: Expander) -> dict:
    a = (C.c_int64 * 10)()
    _check(load_library().relaygr_expander_stats(ex.handle, a))
    return dict(zip(EXPANDER_STATS, list(a)))


# ---- sequence-aware trigger (host arithmetic only) ---------------------------------------------
def relaygr_admission_budget_compute(q_m: float, model_slots: int, kv_p99_bytes: float, hbm_bytes: float, r1: float,
                                     n_instances: int, r2: float, t_life_s: float) -> dict:
    p = AdmissionParamsC(q_m, model_slots, kv_p99_bytes, hbm_bytes, r1, n_instances, r2, t_life_s)
    b = AdmissionBudgetC()
    _check(load_library().relaygr_admission_budget_compute(C.byref(p), C.byref(b)))
    return {n: getattr(b, n) for n, _ in AdmissionBudgetC._fields_}


def relaygr_slot_throughput(pre_infer_ms: float) -> float:
    return load_library().relaygr_slot_throughput(pre_infer_ms)


class Trigger:
    """relaygr_trigger: the admission gate of one special instance."""

    def __init__(self, budget: dict, len_threshold: int):
        b = AdmissionBudgetC(*[budget[n] for n, _ in AdmissionBudgetC._fields_])
        h = C.c_void_p()
        _check(load_library().relaygr_trigger_create(C.byref(b), len_threshold, C.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            load_library().relaygr_trigger_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def relaygr_trigger_admit(t: Trigger, now_s: float, prefix_len: int) -> int:
    rc = load_library().relaygr_trigger_admit(t.handle, now_s, prefix_len)
    if rc < 0:
        _check(rc)
    return rc


def relaygr_trigger_release(t: Trigger) -> None:
    _check(load_library().relaygr_trigger_release(t.handle))


def relaygr_trigger_stats(t: Trigger) -> dict:
    a, b, c, d = C.c_int64(), C.c_int64(), C.c_int64(), C.c_int64()
    load_library().relaygr_trigger_stats(t.handle, C.byref(a), C.byref(b), C.byref(c), C.byref(d))
    return {"live": a.value, "admitted": b.value, "refused": c.value, "not_at_risk": d.value}


class Batch:
    """Device embeddings + host offsets of one jagged batch, marshalled as relaygr_batch."""

    def __init__(self, batch: dict, dtype: str, device: str = "cuda:0", handles: Optional[Sequence[int]] = None):
        td = _torch_dtype(dtype)
        self.n_users = int(batch["n_users"])
        dv = torch.device(device)

        def emb(a):
            if isinstance(a, torch.Tensor):
                return a
            return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dv).to(td).contiguous()

        self.prefix_emb = emb(batch["prefix_emb"])
        self.suffix_emb = emb(batch["suffix_emb"])
        self.cand_emb = emb(batch["cand_emb"])
        self.prefix_off = np.ascontiguousarray(batch["prefix_off"], dtype=np.int32)
        self.suffix_off = np.ascontiguousarray(batch["suffix_off"], dtype=np.int32)
        self.cand_off = np.ascontiguousarray(batch["cand_off"], dtype=np.int32)
        self.user_ids = np.ascontiguousarray(batch["user_ids"], dtype=np.uint64)
        self.handles = np.zeros(self.n_users, dtype=np.uint64)
        if handles is not None:
            self.set_handles(handles)
        self.n_cands = int(self.cand_off[-1]) if self.n_users else 0

    def set_handles(self, handles: Sequence[int]) -> None:
        self.handles = np.ascontiguousarray(np.asarray(handles, dtype=np.uint64))

    def c_struct(self) -> BatchC:
        def ptr(t):
            return t.data_ptr() if t.numel() else None
        return BatchC(
            self.n_users,
            self.user_ids.ctypes.data_as(C.POINTER(C.c_uint64)),
            self.handles.ctypes.data_as(C.POINTER(C.c_uint64)),
            ptr(self.prefix_emb), self.prefix_off.ctypes.data_as(C.POINTER(C.c_int32)),
            ptr(self.suffix_emb), self.suffix_off.ctypes.data_as(C.POINTER(C.c_int32)),
            ptr(self.cand_emb), self.cand_off.ctypes.data_as(C.POINTER(C.c_int32)),
        )


def relaygr_prefill_prefix(ctx: Context, pool: KvPool, batch: Batch, stream=None) -> None:
    bc = batch.c_struct()
    _check(load_library().relaygr_prefill_prefix(ctx.handle, pool.handle, C.byref(bc), _stream_ptr(stream)))


def relaygr_rank_with_cache(ctx: Context, pool: Optional[KvPool], batch: Batch, scores: Optional[torch.Tensor] = None,
                            stream=None) -> torch.Tensor:
    if scores is None:
        scores = torch.empty(batch.n_cands, dtype=torch.float32, device=ctx.device)
    bc = batch.c_struct()
    _check(load_library().relaygr_rank_with_cache(ctx.handle, pool.handle if pool is not None else None, C.byref(bc),
                                                  scores.data_ptr(), _stream_ptr(stream)))
    return scores


def relaygr_rank_with_cache_static(ctx: Context, pool: Optional[KvPool], batch: Batch, scores: torch.Tensor, stream=None) -> torch.Tensor:
    """relaygr_rank_with_cache on the library's own scratch; `scores` must be given (nothing is allocated)."""
    bc = batch.c_struct()
    _check(load_library().relaygr_rank_with_cache_static(ctx.handle, pool.handle if pool is not None else None, C.byref(bc),
                                                         scores.data_ptr(), _stream_ptr(stream)))
    return scores


def relaygr_static_scratch_bytes() -> int:
    return load_library().relaygr_static_scratch_bytes()


def relaygr_rank_full_recompute(ctx: Context, batch: Batch, scores: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    if scores is None:
        scores = torch.empty(batch.n_cands, dtype=torch.float32, device=ctx.device)
    bc = batch.c_struct()
    _check(load_library().relaygr_rank_full_recompute(ctx.handle, C.byref(bc), scores.data_ptr(), _stream_ptr(stream)))
    return scores
