"""Model calls on a cache held in 4 bits: the layers, verification, drafts, the search and the decoding loops of a context made
with FLAG_KV4.

A key that rounding moves across a border between two codes changes by a whole step, so an oracle that quantises its own keys
would differ by more than rounding.  The references below therefore take the keys and values that the device stored (read back
and checked against the projections on their own) and compute everything else in 64 bits."""
import numpy as np
import pytest
import torch

import datagen
import kv4_ref as ref
import paper_2505_24196_b200 as clasp
from oracle import clasp_oracle as orc
from paper_2505_24196_b200.decode import greedy_autoregressive
from util import Pair, close_hidden, rel_l2, tol_hidden

pytestmark = pytest.mark.gpu

CTX = 64


@pytest.fixture(scope="module", params=["tiny", "small", "mini8b"])
def model(request):
    cfg = datagen.CONFIGS[request.param]
    return Pair(cfg, 256, 160, max_M=3, max_T=2, flags=clasp.FLAG_KV4)


def held(model, kv, layer):
    c = model.cfg
    return [ref.unpack(b[layer].cpu().numpy(), c.n_kv_heads, model.max_ctx, c.head_dim) for b in (kv.k, kv.v)]


def layer_with(cfg, x, w, k, v, pos, first=0):
    """Decoder layer on rows x at positions pos.. with every key and value given: row t sees rows [0, first + t] of k, v.
    Returns the output and the rows' own projections (keys rotated)."""
    T, G, hd = x.shape[0], cfg.n_q_heads // cfg.n_kv_heads, cfg.head_dim
    h = orc.rmsnorm(x, w["attn_norm"], cfg.rms_eps)
    at = np.arange(pos, pos + T)
    q = orc.rope((h @ w["wq"].T).reshape(T, -1, hd), at, cfg.rope_theta)
    own_k = orc.rope((h @ w["wk"].T).reshape(T, -1, hd), at, cfg.rope_theta)
    own_v = (h @ w["wv"].T).reshape(T, -1, hd)
    att, _, _ = ref.attention(q, k, v, np.arange(k.shape[0])[None, :] <= first + np.arange(T)[:, None])
    x = x + att.reshape(T, -1) @ w["wo"].T
    h = orc.rmsnorm(x, w["mlp_norm"], cfg.rms_eps)
    return x + (orc.silu(h @ w["w_gate"].T) * (h @ w["w_up"].T)) @ w["w_down"].T, own_k, own_v


def check_stored(cfg, got, want, tol):
    """Stored values against the projections they come from: half a step of the block, and what the projection itself may be
    off (tol of its root mean square, eight times that for a single value, moved through the scale's own step as well)."""
    blocks = lambda a: a.reshape(a.shape[0], -1, 16)
    g, w = blocks(got), blocks(want)
    off = 8 * tol * np.sqrt(np.mean(want ** 2))
    amax = np.abs(w).max(-1, keepdims=True) + off
    assert (np.abs(g - w) <= amax / 7 * 9 / 8 / 2 + off).all()


def test_contexts_with_such_a_cache_run_one_kernel_per_step(model):
    assert not model.engine.engine_active()


@pytest.mark.parametrize("n", [1, 5, 64, 150])
def test_verification_layer_by_layer(model, n):
    """hidden_out of a prompt and of rows behind it: every layer's output from its input and the stored cache."""
    cfg, eng = model.cfg, model.engine
    kv = clasp.KV4Cache(model.ccfg)
    toks = datagen.token_ids(cfg, CTX + n).cuda()
    eng.verify(toks[:CTX], 0, kv, 0, want_hidden=False)
    _, hid = eng.verify(toks[CTX:], CTX, kv, 1)
    assert eng.device_status() == 0
    hid = hid.double().cpu().numpy()
    tol = tol_hidden(cfg)
    for l in range(cfg.L):
        k, v = held(model, kv, l)
        assert (k[CTX + n:] == 0).all() and (v[CTX + n:] == 0).all()         # rows behind the last stay as they were
        out, own_k, own_v = layer_with(cfg, hid[:, l], model.oracle.layer(l), k[:CTX + n], v[:CTX + n], CTX, CTX)
        check_stored(cfg, k[CTX:CTX + n], own_k, tol)
        check_stored(cfg, v[CTX:CTX + n], own_v, tol)
        assert close_hidden(hid[:, l + 1], out, tol), (l, rel_l2(hid[:, l + 1], out))


def test_one_token_at_a_time_is_the_verification(model):
    """Hidden states and cache bytes of a verification against one-token calls, bit for bit."""
    cfg, eng = model.cfg, model.engine
    toks = datagen.token_ids(cfg, CTX + 6).cuda()
    caches = [clasp.KV4Cache(model.ccfg) for _ in range(2)]
    for kv in caches:
        eng.verify(toks[:CTX], 0, kv, 0, want_hidden=False)
    _, many = eng.verify(toks[CTX:], CTX, caches[0], 6)
    many = many.clone()
    for t in range(6):
        _, one = eng.verify(toks[CTX + t:CTX + t + 1], CTX + t, caches[1], 1)
        assert torch.equal(one[0], many[t]), t
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v, caches[1].v)


@pytest.mark.parametrize("S,T", [(1, 1), (3, 1), (2, 4), (1, 9)])
def test_layer_of_candidate_states(model, S, T):
    """Rows that do not write: their own keys are quantised all the same, states do not see each other, the cache stays."""
    cfg, eng = model.cfg, model.engine
    kv = clasp.KV4Cache(model.ccfg)
    eng.verify(datagen.token_ids(cfg, CTX).cuda(), 0, kv, 0, want_hidden=False)
    x = datagen.normal_rows(17, S, (S * T, cfg.d_model)).float().cuda()
    before = kv.k.clone(), kv.v.clone()
    got = eng.layer_forward(1, x, S, T, CTX, CTX, kv)
    assert torch.equal(kv.k, before[0]) and torch.equal(kv.v, before[1])
    for s in range(S):
        xs = x[s * T:(s + 1) * T].contiguous()
        one = eng.layer_forward(1, xs, 1, T, CTX, CTX, kv)                     # the state alone
        assert rel_l2(got[s * T:(s + 1) * T].cpu().numpy(), one.cpu().numpy()) < tol_hidden(cfg) / 10
        wrote = eng.layer_forward(1, xs, 1, T, CTX, CTX, kv, write_kv=True)    # the same rows, stored
        k, v = held(model, kv, 1)
        want, _, _ = layer_with(cfg, xs.double().cpu().numpy(), model.oracle.layer(1), k[:CTX + T], v[:CTX + T], CTX, CTX)
        assert close_hidden(wrote.cpu().numpy(), want, tol_hidden(cfg))
        assert close_hidden(got[s * T:(s + 1) * T].cpu().numpy(), want, tol_hidden(cfg))


@pytest.mark.parametrize("T", [1, 2])
def test_search_is_the_recursion_over_its_layers(model, T):
    """Eq. 2 replayed on the host with the context's own layer_forward: scores of every cell; the decisions where the two
    candidates' cosines are further apart than rounding, the skip set and g[L][M] when all of them are."""
    cfg, eng, M = model.cfg, model.engine, 3
    L, d = cfg.L, cfg.d_model
    kv = clasp.KV4Cache(model.ccfg)
    toks = datagen.token_ids(cfg, CTX + T).cuda()
    eng.verify(toks[:CTX], 0, kv, 0, want_hidden=False)
    _, hid = eng.verify(toks[CTX:], CTX, kv, 1)            # [T, L + 1, d]
    hid = hid.contiguous()
    res = eng.dp_search(hid, d, (L + 1) * d, kv, CTX, CTX, T, M)
    assert eng.device_status() == 0
    D, margin = res["D"].cpu().numpy(), res["margin"].cpu().numpy()
    x = [hid[:, l].contiguous() for l in range(L + 1)]
    cos = lambda a, b: float(np.mean([orc.cosine_score(a[t].double().cpu().numpy(), b[t].double().cpu().numpy()) for t in range(T)]))
    g, choice = {0: x[0]}, np.full((L + 1, M + 1), 255)
    clear = True
    for i in range(1, L + 1):
        nxt = {0: x[i]}
        assert abs(D[i, 0] - 1.0) < 1e-6
        for j in range(1, min(i, M) + 1):
            skip = g[j - 1]
            if j == i:
                nxt[j], choice[i, j] = skip, orc.SKIP
            else:
                app = eng.layer_forward(i - 1, g[j], 1, T, CTX, CTX, kv)
                m = cos(x[i], app) - cos(x[i], skip)
                assert abs(margin[i, j] - m) < 2e-3
                clear = clear and abs(m) > 4e-3
                take = margin[i, j] > 0
                nxt[j], choice[i, j] = (app, orc.APPLY) if take else (skip, orc.SKIP)
            assert abs(D[i, j] - cos(x[i], nxt[j])) < 1e-3
        g = nxt
    np.testing.assert_array_equal(res["S"].cpu().numpy(), orc.backtrack(choice, L, M))
    assert close_hidden(res["g_final"].cpu().numpy(), g[M].cpu().numpy(), tol_hidden(cfg))


def test_draft_is_the_masked_forward(model):
    """A draft over the kept layers equals those layers applied one by one; skipped layers' caches stay as they are."""
    cfg, eng = model.cfg, model.engine
    kv, kv2 = clasp.KV4Cache(model.ccfg), clasp.KV4Cache(model.ccfg)
    toks = datagen.token_ids(cfg, CTX + 1).cuda()
    eng.verify(toks[:CTX], 0, kv, 0, want_hidden=False)
    kv2.k.copy_(kv.k)
    kv2.v.copy_(kv.v)
    mask = bytes(1 if l in (1, cfg.L - 1) else 0 for l in range(cfg.L))
    out, prob = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda")
    eng.draft_forward(mask, toks[CTX:], CTX, kv, out, prob)
    x = model.head_dev["embed"][toks[CTX:].long()].float()
    for l in range(cfg.L):
        if not mask[l]:
            x = eng.layer_forward(l, x.contiguous(), 1, 1, CTX, CTX, kv2, write_kv=True)
    assert torch.equal(kv.k, kv2.k) and torch.equal(kv.v, kv2.v)
    logits = orc.logits_from_hidden(model.oracle, x.double().cpu().numpy())[0]
    top = np.sort(logits)[-2:]
    assert int(out) == int(orc.argmax_lowest(logits[None])[0]) or top[1] - top[0] < 2e-2 * abs(top[1])
    assert abs(float(prob) - float(orc.top1_probability(logits[None])[0])) < 0.05 * float(prob) + 1e-3


def test_decoding_is_lossless(model):
    """Greedy self-speculative decoding on the 4-bit cache commits the tokens of plain greedy decoding on it."""
    prompt = datagen.token_ids(model.cfg, 40).tolist()
    plain = greedy_autoregressive(model.engine, clasp.KV4Cache(model.ccfg), prompt, 24)
    for M, K in ((0, 3), (2, 4)):
        dec = clasp.SelfSpeculativeDecoder(model.engine, clasp.KV4Cache(model.ccfg), M=M, K=K)
        assert dec.generate(prompt, 24) == plain
    assert model.engine.device_status() == 0


def test_sampling_loop_runs(model):
    prompt = datagen.token_ids(model.cfg, 40).tolist()
    runs = [clasp.SpeculativeSampler(model.engine, clasp.KV4Cache(model.ccfg), M=2, K=3, temperature=1.0, seed=5).generate(prompt, 12)
            for _ in range(2)]
    assert runs[0] == runs[1] and all(0 <= t < model.cfg.vocab for t in runs[0])


def test_moving_a_cache_between_the_two_forms(model):
    """A plain context's prompt moved into a 4-bit cache and back: the values of the format, and decoding goes on from it."""
    cfg = model.cfg
    plain = model.engine_with_flags(0)
    pkv, kv = clasp.KVCache(plain.cfg), clasp.KV4Cache(model.ccfg)
    toks = datagen.token_ids(cfg, CTX + 1).cuda()
    plain.verify(toks[:CTX], 0, pkv, 0, want_hidden=False)
    back = clasp.KVCache(plain.cfg)
    for l in range(cfg.L):
        model.engine.kv4_write(pkv.k[l, :CTX], pkv.v[l, :CTX], 0, kv, layer=l)
        model.engine.kv4_read(0, CTX, kv, layer=l, k_out=back.k[l, :CTX], v_out=back.v[l, :CTX])
        for a, b, p in ((back.k, kv.k, pkv.k), (back.v, kv.v, pkv.v)):
            want = ref.values(*ref.quantise(p[l, :CTX].double().cpu().numpy()))
            np.testing.assert_array_equal(a[l, :CTX].double().cpu().numpy(), want)
    # the plain context over the read-back rows and the 4-bit context over the packed ones: the same cached keys (only the
    # token's own key and value are quantised on one side alone)
    _, a = plain.verify(toks[CTX:], CTX, back, 1)
    _, b = model.engine.verify(toks[CTX:], CTX, kv, 1)
    k, v = held(model, kv, 0)
    want, _, _ = layer_with(cfg, b[:, 0].double().cpu().numpy(), model.oracle.layer(0), k[:CTX + 1], v[:CTX + 1], CTX, CTX)
    assert close_hidden(b[:, 1].double().cpu().numpy(), want, tol_hidden(cfg))
    assert rel_l2(a[:, 1].cpu().numpy(), b[:, 1].cpu().numpy()) < 0.1


@pytest.mark.parametrize("flag", [clasp.FLAG_PRUNE, clasp.FLAG_FORCE_SIMT])
def test_with_the_other_flags(model, flag):
    """The search without its unreachable states, and the CUDA-core products of a bf16 model, on the same kind of cache."""
    cfg, M = model.cfg, 3
    eng = model.engine_with_flags(clasp.FLAG_KV4 | flag)
    kv = clasp.KV4Cache(model.ccfg)
    toks = datagen.token_ids(cfg, CTX + 1).cuda()
    model.engine.verify(toks[:CTX], 0, kv, 0, want_hidden=False)
    _, hid = model.engine.verify(toks[CTX:], CTX, kv, 1)
    hid = hid[0].contiguous()
    a = model.engine.dp_search(hid, cfg.d_model, 0, kv, CTX, CTX, 1, M)
    b = eng.dp_search(hid, cfg.d_model, 0, kv, CTX, CTX, 1, M)
    D, E = a["D"].cpu().numpy(), b["D"].cpu().numpy()
    if flag == clasp.FLAG_PRUNE:
        ok = ~np.isnan(E)
        assert np.array_equal(D[ok], E[ok]) and torch.equal(a["S"], b["S"]) and torch.equal(a["g_final"], b["g_final"])
    else:
        # first cells only: a rounding may move a decision further down
        np.testing.assert_allclose(D[:3], E[:3], atol=1e-3)
    n = 70                               # rows of one launch of the few-row attention and more
    long = datagen.token_ids(cfg, CTX + n).cuda()
    kv2 = clasp.KV4Cache(model.ccfg)
    eng.verify(long[:CTX], 0, kv2, 0, want_hidden=False)
    _, h = eng.verify(long[CTX:], CTX, kv2, 1)
    h = h.double().cpu().numpy()
    k, v = held(model, kv2, 0)
    want, _, _ = layer_with(cfg, h[:, 0], model.oracle.layer(0), k[:CTX + n], v[:CTX + n], CTX, CTX)
    assert close_hidden(h[:, 1], want, tol_hidden(cfg))
    assert eng.device_status() == 0
