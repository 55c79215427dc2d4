"""Calls of the 8-bit cache that are refused, or that arrays changed between calls reach, without a GPU: nothing here gets as far as a launch."""
import ctypes as C
import os
import shutil
import subprocess
import types

import pytest
import torch

import paper_2601_01712_amd as rg


def test_attention_refuses_a_context_on_another_device_than_the_pool():
    cfg = rg.make_config(2, 256, 4, "bf16")
    pool = types.SimpleNamespace(cfg=cfg, dtype="bf16", slab=torch.empty(1), handle=None)
    ctx = types.SimpleNamespace(cfg=cfg, dtype="bf16", scratch=torch.empty(1, device="meta"), handle=None)
    with pytest.raises(rg.RelayGRError) as e:
        rg.relaygr_cache_attend(ctx, pool, 0, rg.KvRows([1], [0, 1]), torch.zeros(1, 256, dtype=torch.bfloat16))
    assert e.value.code == rg.RELAYGR_EINVAL and "context on meta" in str(e.value)


def test_rows_keep_their_offsets_and_take_other_values_in_place():
    """The library reads a KvRows' arrays where they are; the binding checks tensors by their last offset, which therefore stays."""
    rows = rg.KvRows([5, 6], [0, 1, 3], first_token=[10, 20], key_len=[11, 22])
    with pytest.raises(ValueError):
        rows.row_off[-1] = 100
    for name, value in (("row_off", rows.row_off.copy()), ("n_rows", 100), ("n_users", 1), ("handles", rows.handles.copy()), ("first_token", None),
                        ("key_len", rows.key_len + 1)):
        with pytest.raises(AttributeError):
            setattr(rows, name, value)
    assert rows.n_rows == rows.c.row_off[2] == 3
    rows.first_token += 1
    rows.key_len[1] = 23
    rows.handles[0] = 7
    assert [rows.c.first_token[i] for i in range(2)] == [11, 21] and rows.c.key_len[1] == 23 and rows.c.handles[0] == 7


@pytest.mark.parametrize("name", ["relaygr_kv_pool_write", "relaygr_kv_pool_read"])
def test_rows_that_belong_to_no_user_are_refused(name):
    """Offsets start at 0 with no users too: rows before the first user would be returned as nobody wrote them."""
    lib, cfg, handle = rg.load_library(), rg.make_config(2, 256, 4, "bf16"), C.c_void_p()
    assert lib.relaygr_kv_pool_create_q8(C.byref(cfg), C.c_void_p(0x10000000), 1 << 24, 64, C.byref(handle)) == 0

    def call(row_off):
        rows = rg.KvRows([], row_off)
        return getattr(lib, name)(handle, 0, rows.ref, 0x1000, 256, 0x2000, 256, None)
    try:
        assert call([5]) == rg.RELAYGR_EINVAL and "start at 0" in rg.relaygr_last_error()
        assert call([0]) == 0
        none = rg.binding.KvRowsC()
        assert getattr(lib, name)(handle, 0, C.byref(none), None, 256, None, 256, None) == 0
    finally:
        lib.relaygr_kv_pool_destroy(handle)


def test_launches_count_their_threads_in_32_bits(tmp_path):
    """Workgroups of 256 threads: one for each item and head, in eights where an XCD has no head of its own."""
    if shutil.which("g++") is None:
        pytest.skip("no g++")
    lib, src = tmp_path / "attend_launch.so", os.path.join(os.path.dirname(os.path.abspath(__file__)), "attend_launch_shim.cpp")
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", src, "-o", str(lib)], check=True)
    shim = C.CDLL(str(lib))
    shim.attend_groups_of.argtypes, shim.attend_groups_of.restype = [C.c_int64, C.c_int], C.c_int64
    shim.attend_fits_in.argtypes = [C.c_int64, C.c_int]
    for heads in (1, 2, 4, 8, 16, 32):
        for items in (1, 2, 7, 8, 9, 1000, (1 << 24) // heads - 8, (1 << 24) // heads, (1 << 31) // 32, 1 << 40):
            groups = shim.attend_groups_of(items, heads)
            assert groups >= items * heads and groups % min(8, max(heads, 8)) == 0 and groups - items * heads < 8
            assert bool(shim.attend_fits_in(items, heads)) == (groups * 256 < 1 << 32)
        # 32 rows an item: fewer than 2^29 / heads rows of one user fit uncut, save for the last few items
        assert shim.attend_fits_in((1 << 24) // heads - 8, heads) and not shim.attend_fits_in((1 << 24) // heads, heads)
