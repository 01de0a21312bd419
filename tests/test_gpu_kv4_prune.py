"""CLASP_FLAG_PRUNE on a context with a 4-bit cache: the cells from which (L, M) can be reached are the same bits, whatever number
of states the last steps would be left with; the others read NaN."""
import dataclasses

import numpy as np
import pytest
import torch

import datagen
import paper_2505_24196_b200 as clasp
from util import Pair

pytestmark = pytest.mark.gpu


def reachable(L, M):
    """Cells of the table a search without the flag fills, and those it fills with the flag."""
    i, j = np.indices((L + 1, M + 1))
    return j <= i, (j <= i) & ((j == 0) | (j >= M - (L - i)))


@pytest.mark.parametrize("name,L,M,T", [("mini8b", 8, 6, 1), ("mini8b", 8, 7, 2), ("mini8b", 4, 4, 1), ("small", 9, 6, 1),
                                        ("small", 9, 7, 3), ("tiny", 8, 6, 2)])
@pytest.mark.parametrize("ctx", [64, 1500])
def test_pruned_search_is_the_same_bits(name, L, M, T, ctx):
    """Groups of four query heads: steps of five states and more take the kernel of many pairs, the pruned last ones would not."""
    cfg = dataclasses.replace(datagen.CONFIGS[name], name=f"{name}-l{L}", L=L)
    p = Pair(cfg, 2048, 256, max_M=M, max_T=3, flags=clasp.FLAG_KV4)
    pruned = p.engine_with_flags(clasp.FLAG_KV4 | clasp.FLAG_PRUNE)
    kv = clasp.KV4Cache(p.ccfg)
    toks = datagen.token_ids(cfg, ctx + T).cuda()
    for s in range(0, ctx, 256):
        p.engine.verify(toks[s:min(s + 256, ctx)], s, kv, 0, want_hidden=False)
    _, hid = p.engine.verify(toks[ctx:], ctx, kv, 1)
    hid = hid.contiguous()
    d = cfg.d_model
    a, b = (e.dp_search(hid, d, (L + 1) * d, kv, ctx, ctx, T, M) for e in (p.engine, pruned))
    assert p.engine.device_status() == 0 and pruned.device_status() == 0
    every, kept = reachable(L, M)
    for key in ("D", "margin"):
        x, y = a[key].cpu().numpy(), b[key].cpu().numpy()
        if key == "D":
            assert (np.isfinite(x) == every).all() and (np.isfinite(y) == kept).all()
        else:
            assert np.isnan(y[~kept]).all()
        np.testing.assert_array_equal(x[kept], y[kept])
    assert torch.equal(a["S"], b["S"]) and torch.equal(a["g_final"], b["g_final"])
    # and with decisions that are given
    forced = torch.randint(0, 2, (L + 1, M + 1), generator=torch.Generator().manual_seed(L * M), dtype=torch.uint8).cuda()
    a, b = (e.dp_search(hid, d, (L + 1) * d, kv, ctx, ctx, T, M, forced_choice=forced) for e in (p.engine, pruned))
    np.testing.assert_array_equal(a["D"].cpu().numpy()[kept], b["D"].cpu().numpy()[kept])
    assert torch.equal(a["S"], b["S"]) and torch.equal(a["g_final"], b["g_final"])
