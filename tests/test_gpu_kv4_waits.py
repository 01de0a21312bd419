"""Waits of the attention of many rows over a 4-bit cache under a limit of a few polls: they run out on a healthy call, the call
ends by itself and says so once, and the next call with the usual limit gives the bits of before."""
import pytest
import torch

from test_gpu_kv4 import make, rows

pytestmark = pytest.mark.gpu

TIMEOUT = -6


@pytest.mark.parametrize("heads,T,ctx", [((32, 8, 128), 20, 40000), ((32, 8, 128), 100, 40000), ((8, 2, 64), 100, 3000),
                                         ((8, 2, 64), 300, 0), ((32, 8, 128), 400, 0)])
def test_waits_that_run_out_are_reported_every_time(heads, T, ctx):
    """One and two blocks of pairs per CTA, keys in parts that are joined and in one, both head dimensions."""
    n_q, n_kv, hd = heads
    eng, kv = make(heads, ctx + T + 8, max_rows=T)
    eng.kv4_write(rows(1, (ctx + T, n_kv, hd), "bf16").cuda(), rows(2, (ctx + T, n_kv, hd), "bf16").cuda(), 0, kv)
    q = rows(3, (T, n_q, hd), "bf16").cuda()
    want = eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx).clone()
    assert eng.device_status() == 0
    # queries take longer to arrive than one poll, and every tile's weights do
    for polls in (1, 1, 1):
        eng.set_wait_limit(polls)
        eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx)
        assert eng.device_status() == TIMEOUT, polls
        assert eng.device_status() == 0            # said once
        eng.set_wait_limit(0)
        assert torch.equal(eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx), want)
        assert eng.device_status() == 0
    # limits that run out somewhere inside the call, with multiplies in flight, or not at all
    for polls in (2, 3, 5, 8, 12, 20, 40, 80):
        eng.set_wait_limit(polls)
        eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx)
        assert eng.device_status() in (0, TIMEOUT)
        assert eng.device_status() == 0
        eng.set_wait_limit(0)
        assert torch.equal(eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx), want)
    # a limit far above what the call needs leaves its bits alone
    eng.set_wait_limit(1 << 20)
    assert torch.equal(eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx), want)
    assert eng.device_status() == 0
