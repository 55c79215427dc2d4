"""Calls of the 8-bit cache that are refused, or that arrays changed between calls reach, without a GPU: nothing here gets as far as a launch."""
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
