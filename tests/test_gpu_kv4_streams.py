"""Results and caches on a context whose stream is not the current one: memory that the current stream still works on is not
written to, and a new cache is ready."""
import pytest
import torch

import datagen
import paper_2505_24196_b200 as clasp
from test_gpu_kv4 import rows
from util import Pair

pytestmark = pytest.mark.gpu

SLEEP = 50_000_000      # clock cycles that the current stream is kept busy for: some 25 ms


def on_a_stream(flags=clasp.FLAG_KV4, cap=64):
    cfg = clasp.ClaspConfig(L=1, d_model=1024, n_q_heads=8, n_kv_heads=2, head_dim=128, d_ffn=8, vocab=8, dtype=clasp.CLASP_BF16,
                            rms_eps=1e-5, rope_theta=5e5, max_ctx=cap, max_rows=64, max_M=0, max_T=1, max_head_rows=1, flags=flags)
    eng = clasp.Clasp(cfg, stream=torch.cuda.Stream())
    return eng, cfg


def busy_blocks(*tensors):
    """Memory of the given kind that goes back to the current stream's pool while a late fill of it is queued."""
    late = [torch.empty_like(t) for t in tensors for _ in range(4)]
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    for t in late:
        t.fill_(7)


def test_results_do_not_lie_in_memory_the_current_stream_still_fills():
    eng, cfg = on_a_stream()
    kv = clasp.KV4Cache(cfg)
    k, v = rows(1, (40, 2, 128), "bf16").cuda(), rows(2, (40, 2, 128), "bf16").cuda()
    q = rows(3, (40, 8, 128), "bf16").cuda()
    torch.cuda.synchronize()
    eng.kv4_write(k, v, 0, kv)
    want = eng.kv4_attention(q, kv, 40)
    want_k, want_v = eng.kv4_read(0, 40, kv)
    torch.cuda.synchronize()
    calls = [(lambda: [eng.kv4_attention(q, kv, 40)], [want]), (lambda: eng.kv4_read(0, 40, kv), [want_k, want_v]),
             (lambda: eng.kv4_read(0, 40, kv, k_out=mine)[1:], [want_v])]
    mine = torch.empty_like(k)
    for call, expect in calls:
        call()
        torch.cuda.synchronize()
        busy_blocks(*expect)
        got = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, expect))


def test_results_of_model_calls_on_another_stream():
    cfg = datagen.CONFIGS["small"]
    p = Pair(cfg, 96, 32, max_M=2, flags=clasp.FLAG_KV4)
    eng = clasp.Clasp(p.ccfg, stream=torch.cuda.Stream())
    eng.load_layers(0, p.layers_dev)
    eng.load_head(p.head_dev)
    toks = datagen.token_ids(cfg, 20).cuda()
    kv = clasp.KV4Cache(p.ccfg)
    torch.cuda.synchronize()
    am, hid = eng.verify(toks, 0, kv, 4)
    torch.cuda.synchronize()
    x = hid[:, 1].contiguous()
    torch.cuda.synchronize()
    calls = {"verify": lambda: eng.verify(toks, 0, kv, 4), "layer": lambda: [eng.layer_forward(2, x, 20, 1, 20, 20, kv)],
             "search": lambda: list(eng.dp_search(hid[19], cfg.d_model, 0, kv, 19, 19, 1, 2).values())}
    for name, call in calls.items():
        want = call()
        torch.cuda.synchronize()
        want = [t.clone() for t in want]
        torch.cuda.synchronize()
        busy_blocks(*want)
        got = call()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(torch.nan_to_num(a.float(), nan=-5.0), torch.nan_to_num(b.float(), nan=-5.0)), name


@pytest.mark.parametrize("packed", [True, False])
def test_a_new_cache_is_ready_on_any_stream(packed):
    """The zeros of a cache made while the current stream is busy do not come after the first rows."""
    eng, cfg = on_a_stream(clasp.FLAG_KV4 if packed else 0)
    k, v = rows(1, (40, 2, 128), "bf16").cuda(), rows(2, (40, 2, 128), "bf16").cuda()
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    kv = (clasp.KV4Cache if packed else clasp.KVCache)(cfg)
    if packed:
        eng.kv4_write(k, v, 3, kv)
    else:
        with torch.cuda.stream(eng.stream):
            kv.k[0, 3:43].copy_(k)
    torch.cuda.synchronize()
    if packed:
        other = clasp.KV4Cache(cfg)
        eng.kv4_write(k, v, 3, other)
        torch.cuda.synchronize()
        assert torch.equal(kv.k, other.k) and torch.equal(kv.v, other.v) and bool((kv.k != 0).any())
    else:
        assert torch.equal(kv.k[0, 3:43], k)
