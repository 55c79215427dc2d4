"""The softmax form's rows are means of V: where every key has the same V, each row is that V, whatever its weights are and however many of them
round.  V is exact in e4m3, and numerator and denominator add the same n <= 1000 weights in 32 bits, each off by at most n * 2^-24 of itself: 2^-13
together, less than half a step of either type below a power of two (2^-9, 2^-12).  So the rows are equal to V in every bit."""
import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
from q8_util import TORCH, context_for, model, offsets, pool_for

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def attend_constant(d, heads, dtype, lens, rows, q, k, causal=False):
    """(out, V) of rows q over keys k whose V is one row of powers of two and 1.5 times such."""
    ctx = context_for(model(d, heads, dtype, "softmax"), len(lens), sum(rows))
    pool, handles = pool_for(ctx.cfg, dtype, lens)
    one = torch.tensor([1.0, -1.5, 2.0, -0.5, 0.75, 1.0, 3.0, -1.0]).repeat(d // 8).to(TORCH[dtype]).to(DEV)
    rg.relaygr_kv_pool_write(pool, 1, rg.KvRows(handles, offsets(lens)), k.to(TORCH[dtype]).to(DEV), one.expand(sum(lens), d).contiguous())
    return rg.relaygr_cache_attend(ctx, pool, 1, rg.KvRows(handles, offsets(rows)), q.to(TORCH[dtype]).to(DEV), causal=causal), one


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,heads", [(256, 8), (256, 4), (256, 2)])
def test_rows_whose_weight_is_a_few_keys(d, heads, dtype, causal):
    """Scores far apart: most of a row's weight is one key's that is not the row's reference, and its rounding must not be the row's."""
    rng = np.random.default_rng(heads)
    lens, rows = [1, 40, 70, 64, 130, 600, 1000], [1, 33, 64, 40, 100, 5, 1]
    q, k = (torch.from_numpy(1.6 * rng.standard_normal((n, d)).astype(np.float32)) for n in (sum(rows), sum(lens)))
    out, one = attend_constant(d, heads, dtype, lens, rows, q, k, causal)
    assert torch.equal(out, one.expand_as(out))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d,heads", [(256, 4), (512, 4)])
def test_rows_of_many_weights_below_the_types_normal_ones(d, heads, dtype):
    """One key of weight 1 and 999 of exp(-11), 2^-15.9: subnormal in fp16, and 1.7 % of the row together."""
    dh, n = d // heads, 1000
    q, k = torch.zeros(3, heads, dh), torch.zeros(n, heads, dh)
    q[..., 0] = dh ** 0.5
    k[1:, :, 0] = -11.0
    out, one = attend_constant(d, heads, dtype, [n], [3], q.view(3, d), k.view(n, d))
    assert torch.equal(out, one.expand_as(out))
    k[0, :, 0], k[500, :, 0] = -11.0, 0.0         # the large weight in the middle
    out, _ = attend_constant(d, heads, dtype, [n], [3], q.view(3, d), k.view(n, d))
    assert torch.equal(out, one.expand_as(out))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_launches_of_two_row_blocks(dtype):
    rng = np.random.default_rng(5)
    lens, rows = [70] * 33, [200] * 33
    q, k = (torch.from_numpy(1.6 * rng.standard_normal((n, 512)).astype(np.float32)) for n in (sum(rows), sum(lens)))
    out, one = attend_constant(512, 8, dtype, lens, rows, q, k)
    assert torch.equal(out, one.expand_as(out))
