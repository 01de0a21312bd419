"""The 4-bit key/value cache (contexts made with FLAG_KV4): rows quantised into it, rows read back, attention over it, against
plain 64-bit forms."""
import numpy as np
import pytest
import torch

import kv4_ref as ref
import paper_2505_24196_b200 as clasp

pytestmark = pytest.mark.gpu

HEADS = [(32, 8, 128), (64, 8, 128), (4, 2, 64), (8, 1, 128), (6, 6, 64), (12, 4, 128)]


def make(heads, capacity, max_rows=64, dtype="bf16"):
    n_q, n_kv, hd = heads
    cfg = clasp.ClaspConfig(L=1, d_model=n_q * hd, n_q_heads=n_q, n_kv_heads=n_kv, head_dim=hd, d_ffn=8, vocab=8,
                            dtype=clasp.CLASP_BF16 if dtype == "bf16" else clasp.CLASP_FP32, rms_eps=1e-5, rope_theta=5e5,
                            max_ctx=capacity, max_rows=max_rows, max_M=0, max_T=1, max_head_rows=1, flags=clasp.FLAG_KV4)
    return clasp.Clasp(cfg), clasp.KV4Cache(cfg)


def dt(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def rows(seed, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen(seed)) * scale).to(dt(dtype))


def set_cache(kv, heads, capacity, k, v, pos0=0, fill=0x5A):
    """Packs k, v [n, n_kv, hd] at pos0 by the plain form; every other byte is `fill`.  Returns the stored values."""
    out = []
    for buf, x in ((kv.k, k), (kv.v, v)):
        a = np.full(buf.shape[1], fill, dtype=np.uint8)
        c, b = ref.quantise(ref.to_np(x))
        ref.pack(c, b, a, heads[1], capacity, heads[2], pos0)
        buf[0].copy_(torch.from_numpy(a))
        out.append(ref.values(c, b))
    return out


# ------------------------------------------------------------------ write and read

def special_rows(n, n_kv, hd, dtype, seed):
    """Rows whose blocks reach every corner of the quantiser."""
    x = torch.randn((n, n_kv, hd), generator=gen(seed), dtype=torch.float64)
    x *= torch.exp2(torch.randint(-22, 16, (n, n_kv, hd // 16), generator=gen(seed + 1)).double()).repeat_interleave(16, -1)
    blocks = x.view(-1, 16)
    m = blocks.shape[0]
    pick = torch.randint(0, 9, (m,), generator=gen(seed + 2))
    half_steps = torch.randint(-14, 15, (m, 16), generator=gen(seed + 3)).double() / 2
    half_steps[:, 0] = 7.0                      # the block's scale is exactly s, every other value on a code or on a border
    s = torch.from_numpy(ref.TABLE[torch.randint(1, ref.TOP + 1, (m,), generator=gen(seed + 4)).numpy()])
    blocks[pick == 0] = (half_steps * s[:, None])[pick == 0]
    blocks[pick == 1] = 0.0
    blocks[pick == 2, 3] = float("inf")
    blocks[pick == 3, 15] = float("nan")
    blocks[pick == 4, 7] = -3e30
    blocks[pick == 5] *= 2.0 ** -110
    border = half_steps * s[:, None]
    blocks[pick == 6] = (border * (1 + 2.0 ** -23))[pick == 6]     # fp32: one step beside the borders
    return x.to(dt(dtype))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("n,pos0", [(1, 0), (1, 40), (2, 7), (17, 3), (130, 1)])
def test_write_gives_the_bytes_of_the_definition(heads, dtype, n, pos0):
    cap = pos0 + n + 5
    eng, kv = make(heads, cap, dtype=dtype)
    k, v = (special_rows(n, heads[1], heads[2], dtype, s) for s in (n, n + 100))
    kv.k.fill_(0xA5)
    kv.v.fill_(0xA5)
    # columns of one fused buffer: rows further apart than they are long
    fused = torch.empty((n, 3 * heads[1] * heads[2]), dtype=dt(dtype), device="cuda")
    kd, vd = fused[:, heads[1] * heads[2]:2 * heads[1] * heads[2]].unflatten(1, (-1, heads[2])), \
        fused[:, 2 * heads[1] * heads[2]:].unflatten(1, (-1, heads[2]))
    kd.copy_(k)
    vd.copy_(v)
    eng.kv4_write(kd, vd, pos0, kv)
    k_out, v_out = eng.kv4_read(pos0, n, kv)
    torch.cuda.synchronize()
    for buf, x, back in ((kv.k, k, k_out), (kv.v, v, v_out)):
        want = np.full(buf.shape[1], 0xA5, dtype=np.uint8)
        c, b = ref.quantise(ref.to_np(x))
        ref.pack(c, b, want, heads[1], cap, heads[2], pos0)
        np.testing.assert_array_equal(buf[0].cpu().numpy(), want)
        np.testing.assert_array_equal(ref.to_np(back), ref.values(c, b))     # every value is exact in the model dtype


def test_error_of_a_row_is_at_most_half_a_step():
    eng, kv = make((8, 2, 128), 256)
    x = rows(3, (200, 2, 128), "bf16", 5.0).cuda()
    eng.kv4_write(x, x, 0, kv)
    back, _ = eng.kv4_read(0, 200, kv)
    a = x.float().unflatten(-1, (-1, 16))
    err = (a - back.float().unflatten(-1, (-1, 16))).abs().amax(-1)
    # half a step; the step is the smallest scale with three mantissa bits that is no less than max / 7: at most 9/8 of it
    assert bool((err <= a.abs().amax(-1) / 7 * 9 / 8 / 2).all())


def test_read_every_code_and_scale():
    """All 16 codes under all 256 scale bytes (the writer makes 1..15 and no scale above its largest; a cache from elsewhere
    may hold the rest): the value the definition names, infinite or NaN scales as NaN or infinities."""
    heads, cap = (4, 2, 64), 64
    eng, kv = make(heads, cap, dtype="fp32")
    for buf in (kv.k, kv.v):
        a = np.zeros(buf.shape[1], dtype=np.uint8)
        codes, scales = ref.parts(a, 2, cap, 64)
        codes[:] = np.tile(np.arange(8, dtype=np.uint8) * 2 + ((np.arange(8, dtype=np.uint8) * 2 + 1) << 4), 4)
        scales[:] = np.arange(512).reshape(2, cap, 4) & 255
        buf[0].copy_(torch.from_numpy(a))
    k, v = eng.kv4_read(0, cap, kv)
    with np.errstate(invalid="ignore"):
        table = np.arange(256, dtype=np.uint16) << 7
        want = (np.arange(16) - 8.0) * table.view(np.float16).astype(np.float64)[np.arange(512).reshape(2, cap, 4) & 255][..., None]
    want = want.reshape(2, cap, 64).transpose(1, 0, 2)
    np.testing.assert_array_equal(ref.to_np(k), want)
    np.testing.assert_array_equal(ref.to_np(v), want)


def test_read_into_strided_rows_leaves_the_rest():
    heads, cap = (8, 2, 128), 40
    eng, kv = make(heads, cap)
    k, v = rows(1, (30, 2, 128), "bf16"), rows(2, (30, 2, 128), "bf16")
    kk, vv = set_cache(kv, heads, cap, k, v)
    big = torch.full((30, 3 * 256), 7.0, dtype=torch.bfloat16, device="cuda")
    eng.kv4_read(0, 30, kv, k_out=big[:, :256].unflatten(1, (2, 128)), v_out=big[:, 512:].unflatten(1, (2, 128)))
    got = ref.to_np(big)
    np.testing.assert_array_equal(got[:, :256].reshape(30, 2, 128), kk)
    np.testing.assert_array_equal(got[:, 512:].reshape(30, 2, 128), vv)
    assert (got[:, 256:512] == 7.0).all()


# ------------------------------------------------------------------ attention

def attend_case(heads, dtype, S, T, ctx, own, ragged, seed, capacity=None, max_rows=None, own_at=None, qscale=1.0, fill=0xFF):
    """One call against the plain form.  Bytes outside the rows in use read as NaN."""
    n_q, n_kv, hd = heads
    R = S * T
    own_at = ctx if own_at is None else own_at
    cap = capacity or max(ctx, own_at + (R if own else 0)) + 3
    eng, kv = make(heads, cap, max_rows or max(R, 1), dtype)
    k, v = rows(seed, (ctx, n_kv, hd), dtype, 1.5), rows(seed + 1, (ctx, n_kv, hd), dtype)
    kk, vv = set_cache(kv, heads, cap, k, v, fill=fill)
    if own:
        ok, ov = rows(seed + 2, (R, n_kv, hd), dtype, 1.5), rows(seed + 3, (R, n_kv, hd), dtype)
        eng.kv4_write(ok.cuda(), ov.cuda(), own_at, kv)
        kk = np.concatenate((kk, ref.values(*ref.quantise(ref.to_np(ok)))))
        vv = np.concatenate((vv, ref.values(*ref.quantise(ref.to_np(ov)))))
    vis = None
    if ragged:
        vis = torch.randint(-2, ctx + 3, (R,), generator=gen(seed + 5), dtype=torch.int32)
        vis[::3] = 0
    q = rows(seed + 4, (R, n_q, hd), dtype, qscale)
    fused = torch.zeros((R, (n_q + 2) * hd), dtype=dt(dtype), device="cuda")
    qd = fused[:, :n_q * hd].unflatten(1, (n_q, hd))
    qd.copy_(q)
    out = torch.full((R, (n_q + 1) * hd), 9.0, dtype=dt(dtype), device="cuda")
    od = out[:, :n_q * hd].unflatten(1, (n_q, hd))
    eng.kv4_attention(qd, kv, ctx, T=T, own_pos0=own_at if own else None, visible=None if vis is None else vis.cuda(), out=od)
    assert eng.device_status() == 0
    want, spread, vmax = ref.attention(ref.to_np(q), kk, vv, ref.seen_mask(R, T, ctx, own, vis))
    got = ref.to_np(od)
    tol = ref.tolerance(want, spread, vmax, dtype == "bf16")
    err = np.abs(got - want)
    assert (err <= tol).all(), (float((err / np.maximum(tol, 1e-30)).max()), np.argwhere(~(err <= tol))[:4])
    assert bool((out[:, n_q * hd:] == 9.0).all())
    return eng, kv, qd, od


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 17, 127, 129, 700])
def test_one_token(heads, dtype, ctx):
    attend_case(heads, dtype, 1, 1, ctx, True, False, seed=ctx)
    if ctx:
        attend_case(heads, dtype, 1, 1, ctx, False, False, seed=ctx + 1)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,S,T,ctx,own_at", [
    ((32, 8, 128), 1, 5, 300, None),       # verification
    ((64, 8, 128), 1, 7, 33, None),
    ((32, 8, 128), 12, 1, 260, None),      # states of a search, their rows parked behind the context
    ((32, 8, 128), 4, 3, 90, 128),         # ... and further away
    ((8, 1, 128), 3, 5, 129, None),
    ((4, 2, 64), 1, 33, 64, None),
    ((6, 6, 64), 9, 2, 50, None),
    ((12, 4, 128), 1, 64, 0, None),        # nothing before the rows
    ((12, 4, 128), 2, 40, 17, 70),
    ((12, 4, 128), 1, 30, 40, 60),         # one state, its rows not behind the context
])
def test_rows_with_their_own_keys(heads, dtype, S, T, ctx, own_at):
    attend_case(heads, dtype, S, T, ctx, True, False, seed=S * 100 + T, own_at=own_at)


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (12, 4, 128), (8, 1, 128)])
@pytest.mark.parametrize("T,ctx", [(17, 0), (17, 1), (33, 63), (64, 64), (65, 65), (129, 10), (200, 333)])
def test_many_rows(heads, T, ctx):
    """Prompt chunks: blocks of pairs and tiles of keys that end anywhere, whole and cut into parts."""
    attend_case(heads, "bf16", 1, T, ctx, True, False, seed=T + ctx, max_rows=T + 1)
    if ctx:
        attend_case(heads, "bf16", 1, T, ctx, False, False, seed=T + ctx + 1)


def test_a_prompt_of_many_blocks():
    attend_case((32, 8, 128), "bf16", 1, 1100, 5, True, False, seed=9)
    attend_case((8, 2, 64), "bf16", 2, 600, 70, True, False, seed=10)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,R,ctx", [((32, 8, 128), 6, 300), ((4, 2, 64), 33, 1000), ((12, 4, 128), 100, 130), ((8, 1, 128), 1, 40)])
@pytest.mark.parametrize("own", [False, True])
def test_rows_that_see_prefixes_of_their_own(heads, dtype, R, ctx, own):
    """Lengths from below zero to beyond the context; rows that see nothing give zeros."""
    eng, kv, q, out = attend_case(heads, dtype, R, 1, ctx, own, True, seed=R)
    if not own:
        assert bool((out[::3] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("capacity", [5000, 40000])
def test_many_runs_and_few(dtype, capacity):
    """The keys of a position are cut by the capacity: many short runs or a part of one."""
    attend_case((32, 8, 128), dtype, 1, 2, 4500, True, False, seed=5, capacity=capacity)
    attend_case((4, 2, 64), dtype, 3, 1, 3001, True, False, seed=6, capacity=capacity)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("qscale", [1e-30, 1e-3, 30.0])
def test_flat_and_peaked_rows(dtype, qscale):
    attend_case((8, 2, 128), dtype, 1, 3, 200, True, False, seed=8, qscale=qscale)


@pytest.mark.parametrize("R", [2, 40])
def test_a_growing_maximum(R):
    """Scores that rise along the keys move the running maximum at every step."""
    heads, cap = (8, 2, 128), 600
    eng, kv = make(heads, cap)
    k = torch.zeros((512, 2, 128))
    k[:, :, 0] = torch.arange(512).view(-1, 1) / 8.0
    k = k.bfloat16()
    v = rows(2, (512, 2, 128), "bf16")
    kk, vv = set_cache(kv, heads, cap, k, v)
    q = torch.zeros((R, 8, 128))
    q[..., 0] = 20.0
    q[1::2, ..., 0] = -20.0
    q = q.bfloat16()
    out = eng.kv4_attention(q.cuda(), kv, 512)
    want, spread, vmax = ref.attention(ref.to_np(q), kk, vv, ref.seen_mask(R, 1, 512, False))
    assert (np.abs(ref.to_np(out) - want) <= ref.tolerance(want, spread, vmax, True)).all()


@pytest.mark.parametrize("dtype,T", [("bf16", 5), ("fp32", 5), ("bf16", 40)])
def test_nan_blocks_reach_the_rows_that_see_them_only(dtype, T):
    """A NaN in a later row's key or value leaves the earlier rows of the verification as they are; in a visible key it makes the
    whole (row, head) NaN, in a visible value the block's dims."""
    heads, ctx = (8, 2, 128), 37
    eng, kv = make(heads, 128, dtype=dtype)
    k, v = rows(1, (ctx + T, 2, 128), dtype), rows(2, (ctx + T, 2, 128), dtype)
    q = rows(3, (T, 8, 128), dtype).cuda()
    eng.kv4_write(k.cuda(), v.cuda(), 0, kv)
    clean = eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx).clone()
    v[ctx + 3, 1, 70] = float("nan")        # value of row 3, kv head 1, dims 64..79
    k[ctx + 4, 0, 5] = float("inf")         # key of row 4, kv head 0
    eng.kv4_write(k.cuda(), v.cuda(), 0, kv)
    got = eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx)
    nan = torch.isnan(got)
    want = torch.zeros_like(nan)
    want[3:, 4:, 64:80] = True
    want[4:, :4, :] = True
    assert bool((nan == want).all())
    assert bool((got[~want] == clean[~want]).all())
    # the same blocks in the own rows of another state: nothing of them reaches the rows before or behind
    got = eng.kv4_attention(q, kv, ctx, T=1, own_pos0=ctx)
    nan, want = torch.isnan(got), torch.zeros_like(nan)
    want[3, 4:, 64:80] = True
    want[4, :4, :] = True
    assert bool((nan == want).all())


@pytest.mark.parametrize("R", [3, 50])
def test_a_query_that_is_not_finite(R):
    heads = (8, 2, 128)
    eng, kv = make(heads, 64)
    k, v = rows(1, (50, 2, 128), "bf16"), rows(2, (50, 2, 128), "bf16")
    set_cache(kv, heads, 64, k, v)
    q = rows(3, (R, 8, 128), "bf16")
    q[1, 2, 9] = float("inf")
    q[2, 5, 0] = float("nan")
    vis = torch.full((R,), 50, dtype=torch.int32)
    vis[2] = 0
    out = eng.kv4_attention(q.cuda(), kv, 50, visible=vis.cuda())
    nan = torch.isnan(out).cpu()
    want = torch.zeros_like(nan)
    want[1, 2] = True
    assert bool((nan == want).all())
    assert bool((out[2] == 0).all())        # a row that sees nothing, whatever its query


@pytest.mark.parametrize("heads,dtype", [((32, 8, 128), "bf16"), ((64, 8, 128), "bf16"), ((4, 2, 64), "fp32"), ((8, 2, 64), "bf16")])
def test_a_row_is_the_same_bits_whatever_shares_the_call(heads, dtype):
    """Verification rows against one-token calls at their positions: what lossless decoding needs."""
    ctx, T, cap = 777, 7, 4096
    n_q, n_kv, hd = heads
    eng, kv = make(heads, cap, dtype=dtype)
    eng.kv4_write(rows(1, (ctx + T, n_kv, hd), dtype).cuda(), rows(2, (ctx + T, n_kv, hd), dtype).cuda(), 0, kv)
    q = rows(3, (T, n_q, hd), dtype).cuda()
    many = eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx)
    for r in range(T):
        one = eng.kv4_attention(q[r:r + 1], kv, ctx + r, own_pos0=ctx + r)
        assert torch.equal(one[0], many[r]), r


def test_captured_calls_follow_their_inputs():
    """A captured write and attention replayed on new rows and a new visible length; two captured graphs in turn."""
    heads, cap = (32, 8, 128), 2048
    stream = torch.cuda.Stream()
    n_q, n_kv, hd = heads
    with torch.cuda.stream(stream):
        eng, kv = make(heads, cap)
        k, v = rows(1, (1000, n_kv, hd), "bf16").cuda(), rows(2, (1000, n_kv, hd), "bf16").cuda()
        eng.kv4_write(k, v, 0, kv)
        q = torch.zeros((1, n_q, hd), dtype=torch.bfloat16, device="cuda")
        vis = torch.zeros(1, dtype=torch.int32, device="cuda")
        outs = [torch.empty_like(q) for _ in range(2)]
        eng.kv4_attention(q, kv, cap, visible=vis, out=outs[0])
        stream.synchronize()
        graphs = []
        for o in outs:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=stream):
                eng.kv4_attention(q, kv, cap, visible=vis, out=o)
            graphs.append(g)
        for n in (1, 17, 500, 1000):
            q.copy_(rows(n, (1, n_q, hd), "bf16"))
            vis.fill_(n)
            graphs[0].replay()
            graphs[1].replay()
            want = eng.kv4_attention(q, kv, cap, visible=vis)
            stream.synchronize()
            assert torch.equal(outs[0], want) and torch.equal(outs[1], want)
            full, spread, vmax = ref.attention(ref.to_np(q), ref.unpack(kv.k[0].cpu().numpy(), n_kv, cap, hd)[:n],
                                               ref.unpack(kv.v[0].cpu().numpy(), n_kv, cap, hd)[:n], np.ones((1, n), bool))
            assert (np.abs(ref.to_np(want) - full) <= ref.tolerance(full, spread, vmax, True)).all()


@pytest.mark.parametrize("R,own", [(40, False), (24, True)])
def test_captured_calls_of_many_rows(R, own):
    """Attention of many rows, its keys cut into parts and joined, captured once and replayed on new inputs."""
    heads, cap, ctx = (32, 8, 128), 2048, 1500
    stream = torch.cuda.Stream()
    n_q, n_kv, hd = heads
    with torch.cuda.stream(stream):
        eng, kv = make(heads, cap)
        q = torch.zeros((R, n_q, hd), dtype=torch.bfloat16, device="cuda")
        out = torch.empty_like(q)
        call = lambda o: eng.kv4_attention(q, kv, ctx, own_pos0=ctx if own else None, out=o)
        call(out)
        stream.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            eng.kv4_attention(q, kv, ctx, own_pos0=ctx if own else None, out=out)
        for seed in (1, 2):
            q.copy_(rows(seed, (R, n_q, hd), "bf16"))
            eng.kv4_write(rows(seed + 5, (ctx + R, n_kv, hd), "bf16").cuda(), rows(seed + 7, (ctx + R, n_kv, hd), "bf16").cuda(), 0, kv)
            g.replay()
            g.replay()
            want = call(torch.empty_like(q))
            stream.synchronize()
            assert torch.equal(out, want)
            kk, vv = (ref.unpack(b[0].cpu().numpy(), n_kv, cap, hd)[:ctx + (R if own else 0)] for b in (kv.k, kv.v))
            full, spread, vmax = ref.attention(ref.to_np(q), kk, vv, ref.seen_mask(R, 1, ctx, own))
            assert (np.abs(ref.to_np(want) - full) <= ref.tolerance(full, spread, vmax, True)).all()


def test_positions_past_four_gigabytes():
    """A cache whose byte offsets need more than 32 bits: rows at its end are written, read and attended to."""
    heads, cap = (8, 8, 128), 9_000_000        # 4.6 GB of key codes
    eng, kv = make(heads, cap, max_rows=4)
    assert kv.k.shape[1] > 1 << 32
    at = cap - 20
    k, v = rows(1, (20, 8, 128), "bf16"), rows(2, (20, 8, 128), "bf16")
    eng.kv4_write(k.cuda(), v.cuda(), at, kv)
    k_out, v_out = eng.kv4_read(at, 20, kv)
    kk, vv = (ref.values(*ref.quantise(ref.to_np(x))) for x in (k, v))
    np.testing.assert_array_equal(ref.to_np(k_out), kk)
    np.testing.assert_array_equal(ref.to_np(v_out), vv)
    q = rows(3, (4, 8, 128), "bf16")
    out = eng.kv4_attention(q.cuda(), kv, 0, T=4, own_pos0=at + 16)
    want, spread, vmax = ref.attention(ref.to_np(q), kk[16:], vv[16:], np.tril(np.ones((4, 4), bool)))
    assert (np.abs(ref.to_np(out) - want) <= ref.tolerance(want, spread, vmax, True)).all()
    # the whole cache: zero keys but the last twenty, which a large query picks out
    q = torch.zeros((1, 8, 128))
    q[0] = k[-1].float() * 40.0
    q = q.bfloat16()
    out = ref.to_np(eng.kv4_attention(q.cuda(), kv, cap))
    for h in range(8):
        s = kk[:, h] @ ref.to_np(q)[0, h] / np.sqrt(128.0)
        m = max(s.max(), 0.0)
        p = np.exp(s - m)
        want = p @ vv[:, h] / (p.sum() + (cap - 20) * np.exp(-m))
        spread = (np.abs(kk[:, h]) @ np.abs(ref.to_np(q)[0, h])).max() / np.sqrt(128.0)
        assert (np.abs(out[0, h] - want) <= ref.tolerance(want, spread, np.abs(vv).max(), True)).all()


@pytest.mark.parametrize("T", [20, 100])
def test_waits_that_run_out_are_reported(T):
    """The attention of many rows with a wait limit of a few polls: it ends by itself, the status says so once, and the next
    call with the usual limit gives the same bits as before.  (A poll may itself last for microseconds, so a call may also get
    through; the cache comes from memory to make that less likely.)"""
    heads, ctx, cap = (32, 8, 128), 40000, 41000
    eng, kv = make(heads, cap, max_rows=128)
    n_q, n_kv, hd = heads
    eng.kv4_write(rows(1, (ctx + T, n_kv, hd), "bf16").cuda(), rows(2, (ctx + T, n_kv, hd), "bf16").cuda(), 0, kv)
    q = rows(3, (T, n_q, hd), "bf16").cuda()
    flush = torch.empty(256 << 20, dtype=torch.uint8, device="cuda")
    want = eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx).clone()
    assert eng.device_status() == 0
    seen = []
    for polls in (1, 1, 1, 2, 3, 20):
        flush.zero_()
        eng.set_wait_limit(polls)
        eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx)
        seen.append(eng.device_status())
        assert seen[-1] in (0, -6)
        eng.set_wait_limit(0)
        assert eng.device_status() == 0
        assert torch.equal(eng.kv4_attention(q, kv, ctx, T=T, own_pos0=ctx), want)
    print("status under 1, 1, 1, 2, 3, 20 polls:", seen)


# ------------------------------------------------------------------ refusals

def test_refusals_on_the_device():
    heads, cap = (8, 2, 128), 32
    eng, kv = make(heads, cap, max_rows=4)
    lib, h, layer = eng.lib, eng.handle, kv.array[0]
    x = torch.zeros((8, 8, 128), dtype=torch.bfloat16, device="cuda")
    p = x.data_ptr()
    INV, CAP = -1, -3
    w = lambda k=p, ks=256, v=p, vs=256, n=2, pos=0, kvl=layer: lib.clasp_kv4_write(h, k, ks, v, vs, n, pos, kvl)
    r = lambda pos=0, n=2, k=p, ks=256, v=p, vs=256: lib.clasp_kv4_read(h, layer, pos, n, k, ks, v, vs)
    a = lambda q=p, qs=1024, S=1, T=1, c=4, own=-1, vis=None, o=p, os=1024: lib.clasp_kv4_attention(h, q, qs, S, T, c, own, vis, layer, o, os)
    assert w() == r() == a() == 0
    assert w(n=0, k=None) == r(n=0) == a(S=0) == a(T=0) == 0
    for f in (w, r):
        assert f(n=-1) == f(pos=-1) == f(k=None) == f(v=None) == f(k=p + 2) == f(ks=128) == f(vs=260) == INV
        assert f(n=33) == f(pos=31) == f(pos=2 ** 31 - 1) == CAP
    assert a(S=-1) == a(T=-1) == a(c=-1) == a(own=-2) == a(q=None) == a(o=None) == a(o=p + 8) == a(qs=1020) == a(os=512) == a(vis=p + 2) == INV
    assert a(S=5) == a(c=33) == a(own=32) == a(S=65536, T=65536) == CAP
    assert w(kvl=clasp.ClaspKvLayer(None, layer.v)) == w(kvl=clasp.ClaspKvLayer(layer.k + 8, layer.v)) == INV
    assert eng.device_status() == 0
    plain = clasp.ClaspConfig.from_buffer_copy(eng.cfg)
    plain.flags = 0
    other = clasp.Clasp(plain)
    assert lib.clasp_kv4_write(other.handle, p, 256, p, 256, 1, 0, layer) == INV
    assert lib.clasp_kv4_attention(other.handle, p, 1024, 1, 1, 4, -1, None, layer, p, 1024) == INV


def test_refusals_of_the_binding():
    eng, kv = make((8, 2, 128), 32, max_rows=4)
    k, q = torch.zeros((2, 2, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((2, 8, 128), dtype=torch.bfloat16, device="cuda")
    for bad in (k.float(), k.cpu(), k[:, :1], k[..., :64], k.transpose(1, 2).contiguous().transpose(1, 2), k[0]):
        with pytest.raises(ValueError):
            eng.kv4_write(bad, k, 0, kv)
    with pytest.raises(ValueError):
        eng.kv4_write(k, k[:1], 0, kv)
    with pytest.raises(ValueError):
        eng.kv4_write(k, k, 0, kv, layer=1)
    with pytest.raises(ValueError):
        eng.kv4_attention(q, kv, 4, T=3)
    with pytest.raises(ValueError):
        eng.kv4_attention(q, kv, 4, visible=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        eng.kv4_attention(q, kv, 4, own_pos0=-1)
    with pytest.raises(ValueError):
        eng.kv4_attention(q, kv, 4, out=q[:1])
    for call in (lambda: eng.kv4_write(k, k, 1 << 32, kv), lambda: eng.kv4_read(-(1 << 32), 1, kv),
                 lambda: eng.kv4_attention(q, kv, (1 << 32) + 4), lambda: eng.kv4_attention(q, kv, 4, own_pos0=1 << 33)):
        with pytest.raises(ValueError):
            call()
    # a cache of another kind or layout
    other = clasp.KV4Cache(make((8, 2, 128), 31)[0].cfg)
    plain = clasp.ClaspConfig.from_buffer_copy(eng.cfg)
    plain.flags = 0
    for bad in (other, clasp.KVCache(plain)):
        with pytest.raises(ValueError):
            eng.kv4_write(k, k, 0, bad)
        with pytest.raises(ValueError):
            eng.verify(torch.zeros(1, dtype=torch.int32, device="cuda"), 0, bad, 0, want_hidden=False)
    with pytest.raises(ValueError):
        clasp.Clasp(plain).verify(torch.zeros(1, dtype=torch.int32, device="cuda"), 0, kv, 0, want_hidden=False)
    with pytest.raises(clasp.ClaspError):
        eng.kv4_read(31, 2, kv)
    with pytest.raises(ValueError):
        eng.kv4_read(0, -1, kv)
