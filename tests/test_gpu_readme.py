"""The example of README for backbones with their own projections, run as it stands, step after step, against the definitions in 64 bits."""
import ast
import os
import re
import textwrap

import numpy as np
import pytest
import torch

import paper_2601_01712_amd as rg
from q8_util import context_for, model, offsets, pool_for, values
from scored_util import scored, visible

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    with open(os.path.join(ROOT, "README.md")) as f:
        blocks = re.findall(r"(?:^    .*\n)+", f.read(), re.M)
    (code,) = [b for b in blocks if "relaygr_kv_pool_evict" in b]
    return ast.parse(textwrap.dedent(code)).body


def test_a_history_grows_and_is_cut_as_the_readme_says():
    """Every token's weight is the sum of what it itself received, also where it was written to the place of one that left."""
    d, heads, dtype, room, most = 256, 4, "bf16", 512, 300
    dh = d // heads
    rng = np.random.default_rng(31)
    ctx = context_for(model(d, heads, dtype, "softmax"), 2, 256)
    pool, handles = pool_for(ctx.cfg, dtype, [room, room])
    token_off, profile_lens = [0, room], [3, 0]
    ns = dict(rg=rg, np=np, torch=torch, ctx=ctx, cfg=ctx.cfg, pool=pool, layer=1, handles=handles, token_off=token_off, profile_lens=profile_lens,
              weight=torch.zeros(2 * room, device=DEV), key_position=torch.zeros(2 * room, dtype=torch.int32, device=DEV))
    lens, seen = [0, 0], [0, 0]
    total, dtotal = [np.zeros(0), np.zeros(0)], [np.zeros(0), np.zeros(0)]
    evicted = 0
    for step in range(6):
        new = [int(rng.integers(60, 110)), 83]
        row_off, now = offsets(new), [n + m for n, m in zip(lens, new)]
        keep = [min(n, most) for n in now]
        positions = torch.from_numpy(np.concatenate([s + np.arange(m) for s, m in zip(seen, new)]).astype(np.int32)).to(DEV)
        for u in range(2):
            ns["key_position"][token_off[u] + lens[u]:token_off[u] + now[u]] = positions[row_off[u]:row_off[u + 1]]
        ns.update({name: values(rng, sum(new), d, dtype)[0].to(DEV) for name in "qkv"}, positions=positions, row_off=row_off, lengths=lens, lengths_now=now, keep_off=offsets(keep))
        for statement in example():
            exec(compile(ast.Module([statement], []), "README.md", "exec"), ns)
            if "relaygr_cache_attend_scored" not in ast.unparse(statement):
                continue
            for u in range(2):
                q = ns["q"].double().cpu().numpy()[row_off[u]:row_off[u + 1]].reshape(new[u], heads, dh)
                k, v = (x.double().cpu().numpy().reshape(now[u], heads, dh) for x in rg.relaygr_kv_pool_read(pool, 1, rg.KvRows([handles[u]], [0, now[u]])))
                want, bound, t, dt = scored(q, k, v, visible(now[u], new[u], True, profile_lens[u], window=2048), "softmax", dtype, 30.0)
                out = ns["out"][row_off[u]:row_off[u + 1]].double().cpu().numpy().reshape(want.shape)
                assert (np.abs(out - want) <= bound).all(), (step, u)
                total[u] = np.concatenate([total[u], np.zeros(new[u])]) + t
                dtotal[u] = np.concatenate([dtotal[u], np.zeros(new[u])]) + dt + 2.0 ** -23 * total[u]
                got = ns["weight"][token_off[u]:token_off[u] + now[u]].double().cpu().numpy()
                assert (np.abs(got - total[u]) <= dtotal[u]).all(), (step, u)
        kept = ns["kept"].cpu().numpy()
        for u in range(2):
            mine = kept[offsets(keep)[u]:offsets(keep)[u + 1]]
            total[u], dtotal[u] = total[u][mine], dtotal[u][mine]
        evicted += sum(now) - sum(keep)
        lens, seen = keep, [s + m for s, m in zip(seen, new)]
    assert evicted > 0
