"""Attention over a 4-bit cache whose keys are cut into several runs: a row's bits do not depend on the rows that share its call,
on either side of a border between two runs.  (Runs have 1024 keys in all caches here.)"""
import numpy as np
import pytest
import torch

import datagen
import kv4_ref as ref
import paper_2505_24196_b200 as clasp
from paper_2505_24196_b200.decode import greedy_autoregressive
from test_gpu_kv4 import make, rows
from util import Pair

pytestmark = pytest.mark.gpu

RUN, CAP = 1024, 9 * 1024
HEADS = [((64, 8, 128), "bf16"), ((8, 2, 64), "bf16"), ((32, 8, 128), "fp32"), ((4, 2, 64), "fp32")]


def filled(heads, dtype, n, seed=1):
    eng, kv = make(heads, CAP, dtype=dtype)
    k, v = (rows(seed + i, (n,) + heads[1:], dtype).cuda() for i in range(2))
    eng.kv4_write(k, v, 0, kv)
    return eng, kv


@pytest.mark.parametrize("heads,dtype", HEADS)
@pytest.mark.parametrize("border", [1, 2, 4, 6, 8])
@pytest.mark.parametrize("T", [5, 16])
def test_verification_across_a_border(heads, dtype, border, T):
    """Rows that see `border` runs and rows that see one more, in one call and one at a time."""
    ctx = border * RUN - T // 2 - 1
    eng, kv = filled(heads, dtype, ctx + T)
    for seed in range(3, 9):
        q = rows(seed, (T, heads[0], heads[2]), dtype).cuda()
        many = eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx)
        for r in range(T):
            one = eng.kv4_attention(q[r:r + 1], kv, ctx + r, own_pos0=ctx + r)
            assert torch.equal(one[0], many[r]), (seed, r)
    want, spread, vmax = ref.attention(ref.to_np(q), *(ref.unpack(b[0].cpu().numpy(), heads[1], CAP, heads[2])[:ctx + T]
                                                       for b in (kv.k, kv.v)), ref.seen_mask(T, T, ctx, True))
    assert (np.abs(ref.to_np(many) - want) <= ref.tolerance(want, spread, vmax, dtype == "bf16")).all()


@pytest.mark.parametrize("heads,dtype", HEADS)
def test_prefixes_under_a_longer_context(heads, dtype):
    """A row that sees n positions gives the same bits whether the call's context ends there or further on."""
    eng, kv = filled(heads, dtype, CAP)
    ends = [1, 1000, 1024, 1025, 2048, 2049, 3000, 4096, 4097, 5121, 6144, 7000, 8192, 8193]
    vis = torch.tensor(ends, dtype=torch.int32, device="cuda")
    for seed in range(3, 7):
        q = rows(seed, (len(ends), heads[0], heads[2]), dtype).cuda()
        for ctx in (8193, CAP):
            many = eng.kv4_attention(q, kv, ctx, visible=vis)
            for r, n in enumerate(ends):
                assert torch.equal(eng.kv4_attention(q[r:r + 1], kv, n)[0], many[r]), (seed, ctx, n)


@pytest.mark.parametrize("name,border", [("tiny", 4), ("small", 4), ("mini8b", 2), ("mini8b", 4)])
def test_model_calls_across_a_border(name, border):
    """Hidden states, cache bytes and greedy tokens of a model whose verifications straddle a border between runs."""
    cfg = datagen.CONFIGS[name]
    p = Pair(cfg, 8 * 1024, 512, max_M=2, flags=clasp.FLAG_KV4)
    T, ctx = 12, border * RUN - 6
    prompt = datagen.token_ids(cfg, ctx)
    toks = datagen.token_ids(cfg, T, stream=3).cuda()
    caches = [clasp.KV4Cache(p.ccfg) for _ in range(2)]
    for kv in caches:
        for s in range(0, ctx, 512):
            p.engine.verify(prompt[s:s + 512].cuda(), s, kv, 0, want_hidden=False)
    _, many = p.engine.verify(toks, ctx, caches[0], T)
    many = many.clone()
    for t in range(T):
        _, one = p.engine.verify(toks[t:t + 1], ctx + t, caches[1], 1)
        assert torch.equal(one[0], many[t]), t
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)
    prompt = prompt.tolist()
    plain = greedy_autoregressive(p.engine, clasp.KV4Cache(p.ccfg), prompt, 20)
    dec = clasp.SelfSpeculativeDecoder(p.engine, clasp.KV4Cache(p.ccfg), M=2, K=4)
    assert dec.generate(prompt, 20) == plain
    assert p.engine.device_status() == 0
