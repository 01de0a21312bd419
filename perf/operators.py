"""The 4-bit key/value cache and the attention that reads it, as measurable cases.

Three operators: rows quantised into the cache and read back ("store"), rows of a cache read back into the model's type
("read"), attention over the cache ("attend": single tokens, the rows of a verification, the candidate states of a layer
search, a prompt).  The cache format is the library's: a block is 16 consecutive dims of one position's key or value, held as
sixteen 4-bit codes c (low nibble first) and one scale byte b; it stands for (c - 8) * scale(b), where scale(b) is the
half-precision number with the bits b << 7.  One array (keys or values of a layer) is all codes [n_kv, capacity, hd / 2], then
all scale bytes [n_kv, capacity, hd / 16].
"""
import math
import random

import numpy as np
import torch

own = False

BLOCK = 16
TOP_SCALE = 0xC6     # largest scale a block gets (896): 72 * scale stays a finite half-precision number
NAN_SCALE = 0xFF     # a block that held an infinity or NaN


def _case(name, op, dtype, heads, **kw):
    n_q, n_kv, hd = heads
    c = {"name": name, "op": op, "dtype": dtype, "n_q": n_q, "n_kv": n_kv, "hd": hd, "capacity": 0, "rows": 0, "pos0": 0,
         "ctx": 0, "S": 1, "T": 1, "own_rows": False, "ragged": False}
    c.update(kw)
    return c


H8B, H70B, TINY, MINI = (32, 8, 128), (64, 8, 128), (4, 2, 64), (8, 2, 128)


def listed():
    return [
        # one decoded token's keys and values enter the cache of an 8B layer
        _case("store-1", "store", "bf16", H8B, capacity=8192, rows=1, pos0=4999),
        # a prompt chunk of the small fp32 model, an odd number of rows at an odd place
        _case("store-97-fp32", "store", "fp32", TINY, capacity=333, rows=97, pos0=131),
        # a prompt of an 8B layer moved into the 4-bit cache in one go
        _case("store-8192", "store", "bf16", H8B, capacity=8200, rows=8192, pos0=0),
        # part of a small model's cache handed back to the plain path
        _case("read-513", "read", "bf16", MINI, capacity=1024, rows=513, pos0=77),
        # a long context of an 8B layer handed back
        _case("read-32768", "read", "bf16", H8B, capacity=33000, rows=32768, pos0=3),
        # a decoded token over the benchmark's 512-token context (the token itself is in the cache already)
        _case("attend-1-c512", "attend", "bf16", H8B, capacity=1024, ctx=512, own_rows=True),
        # a decoded token at the far end of a long context
        _case("attend-1-c131071", "attend", "bf16", H8B, capacity=131072, ctx=131071, own_rows=True),
        # verification of four drafts and the pending token, 70B heads
        _case("attend-5-c2048-70b", "attend", "bf16", H70B, capacity=4096, ctx=2048, T=5, own_rows=True),
        # the twelve candidate states of a search over the context sweep's longest cache
        _case("attend-12-states-c8192", "attend", "bf16", H8B, capacity=9000, ctx=8192, S=12, own_rows=True),
        # rows of the small fp32 model that see cache prefixes of their own, some of them nothing
        _case("attend-33-ragged-fp32", "attend", "fp32", TINY, capacity=1100, ctx=1000, T=33, ragged=True),
        # a chunk of prompt rows behind a context already in the cache
        _case("attend-128-c4095", "attend", "bf16", H8B, capacity=8192, ctx=4095, T=128, own_rows=True),
        # a ragged prompt in one call
        _case("attend-1999", "attend", "bf16", H8B, capacity=2048, ctx=0, T=1999, own_rows=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["store", "read", "attend", "attend", "attend"])
    heads = rng.choice([H8B, H8B, H70B, TINY, MINI, (8, 2, 64), (12, 4, 128), (6, 6, 64), (8, 1, 128)])
    dtype = "fp32" if heads == TINY else rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op != "attend":
        rows = _log_int(rng, 1, 8000 if op == "store" else 17000)
        pos0 = rng.randint(0, 500)
        return _case("", op, dtype, heads, rows=rows, pos0=pos0, capacity=pos0 + rows + rng.randint(0, 300))
    form = rng.choice(["decode", "decode", "verify", "states", "ragged", "prompt"])
    kw = {"ctx": _log_int(rng, 16, 100000), "own_rows": True}
    if form == "verify":
        kw.update(ctx=_log_int(rng, 16, 32000), T=rng.randint(2, 16))
    elif form == "states":
        kw.update(ctx=_log_int(rng, 16, 12000), S=rng.randint(2, 16), T=rng.choice([1, 1, 2, 4]))
    elif form == "ragged":
        kw.update(ctx=_log_int(rng, 16, 8000), T=rng.randint(1, 60), own_rows=False, ragged=True)
    elif form == "prompt":
        T = _log_int(rng, 65, 1000 if heads == H70B else 1500)
        kw.update(ctx=rng.choice([0, rng.randint(1, 400)]), T=T)
        if dtype == "fp32":
            kw.update(T=min(T, 300))
    c = _case("", "attend", dtype, heads, **kw)
    c["capacity"] = c["ctx"] + c["S"] * c["T"] + rng.randint(0, 500)
    return c


# ------------------------------------------------------------------ inputs

def _dtype(case):
    return torch.float32 if case["dtype"] == "fp32" else torch.bfloat16


def _scales(device):
    """The 256 scale bytes as float32."""
    return (torch.arange(256, dtype=torch.int16, device=device) << 7).view(torch.float16).float()


def _quantise(x):
    """[..., hd] -> (codes uint8 [..., hd / 2], scale bytes uint8 [..., hd / 16]): the smallest scale with 7 * scale >= the
    block's largest magnitude, codes to the nearest (ties to even)."""
    x = x.float().unflatten(-1, (-1, BLOCK))
    table = _scales(x.device)[:TOP_SCALE + 1]
    amax = x.abs().amax(-1)
    byte = torch.bucketize(amax, 7.0 * table).clamp(max=TOP_SCALE)
    s = table[byte].unsqueeze(-1)
    c = torch.where(s > 0, torch.round(x / s).clamp(-7, 7), torch.zeros_like(x))
    bad = ~torch.isfinite(x).all(-1)
    c = torch.where(bad.unsqueeze(-1), torch.zeros_like(c), c) + 8
    byte = torch.where(bad, NAN_SCALE, byte).to(torch.uint8)
    c = c.flatten(-2).to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4), byte


def _dequantise(codes, byte):
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() - 8.0
    return c * _scales(codes.device)[byte.long()].repeat_interleave(BLOCK, -1)


def _split(buf, case):
    """Codes [n_kv, capacity, hd / 2] and scale bytes [n_kv, capacity, hd / 16] of one cache array."""
    n, cap, hd = case["n_kv"], case["capacity"], case["hd"]
    k = n * cap * hd // 2
    return buf[:k].view(n, cap, hd // 2), buf[k:].view(n, cap, hd // BLOCK)


def _rows(gen, case, n, keys):
    """[n, n_kv, hd] as a projection leaves them; keys have a few dims that are larger at every position."""
    x = torch.randn((n, case["n_kv"], case["hd"]), generator=gen, device="cuda")
    if keys:
        w = torch.ones((case["n_kv"], case["hd"]), device="cuda")
        w[:, torch.randperm(case["hd"], generator=gen, device="cuda")[:4]] = 4.0
        x = x * w
    return x


def _inputs(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt, n_q, n_kv, hd = _dtype(case), case["n_q"], case["n_kv"], case["hd"]
    d = {}
    n = case["rows"] if case["op"] != "attend" else case["S"] * case["T"]
    if case["op"] != "read":
        # queries, keys and values of the rows are columns of one projection's output
        qkv = torch.empty((n, (n_q + 2 * n_kv) * hd), dtype=dt, device="cuda")
        q, k, v = (t.unflatten(1, (-1, hd)) for t in qkv.split([n_q * hd, n_kv * hd, n_kv * hd], 1))
        q.copy_(torch.randn((n, n_q, hd), generator=gen, device="cuda"))
        k.copy_(_rows(gen, case, n, True))
        v.copy_(_rows(gen, case, n, False))
        d.update(q=q, k=k, v=v)
    if case["op"] != "store":
        # the cache as earlier calls left it; what lies behind the rows in use is whatever the memory held
        first, used = (0, case["ctx"]) if case["op"] == "attend" else (case["pos0"], case["rows"])
        total = n_kv * case["capacity"] * hd * 9 // 16
        for name, keys in (("kbuf", True), ("vbuf", False)):
            buf = torch.randint(0, 256, (total,), generator=gen, dtype=torch.uint8, device="cuda")
            codes, byte = _split(buf, case)
            parts = [(first, _rows(gen, case, used, keys).to(dt))] if used else []
            if case["own_rows"]:
                parts.append((case["ctx"], d["k" if keys else "v"]))
            for at, x in parts:
                c, b = _quantise(x.transpose(0, 1))
                codes[:, at:at + x.shape[0]], byte[:, at:at + x.shape[0]] = c, b
            d[name] = buf
    if case["ragged"]:
        vis = torch.randint(0, case["ctx"] + 1, (n,), generator=gen, device="cuda", dtype=torch.int32)
        vis[::4] = 0
        d["visible"] = vis
    return d


def prepare(case, seed):
    state = {"case": case}
    state.update(_inputs(case, seed))
    if not own:
        if case["op"] == "store":
            state["kbuf"], state["vbuf"] = (torch.zeros(case["n_kv"] * case["capacity"] * case["hd"] * 9 // 16,
                                                        dtype=torch.uint8, device="cuda") for _ in range(2))
        return state
    import paper_2505_24196_b200 as clasp
    cfg = clasp.ClaspConfig(L=1, d_model=case["n_q"] * case["hd"], n_q_heads=case["n_q"], n_kv_heads=case["n_kv"],
                            head_dim=case["hd"], d_ffn=8, vocab=8,
                            dtype=clasp.CLASP_FP32 if case["dtype"] == "fp32" else clasp.CLASP_BF16, rms_eps=1e-5,
                            rope_theta=500000.0, max_ctx=case["capacity"], max_rows=max(case["S"] * case["T"], 1), max_M=0,
                            max_T=1, max_head_rows=1, flags=clasp.FLAG_KV4)
    state["engine"] = clasp.Clasp(cfg)
    state["kv"] = clasp.KV4Cache(cfg)
    if case["op"] != "store":
        state["kv"].k[0].copy_(state.pop("kbuf"))
        state["kv"].v[0].copy_(state.pop("vbuf"))
    return state


# ------------------------------------------------------------------ one pass

def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    case, eng, kv = state["case"], state["engine"], state["kv"]
    if case["op"] == "store":
        eng.kv4_write(state["k"], state["v"], case["pos0"], kv)
    if case["op"] != "attend":
        return eng.kv4_read(case["pos0"], case["rows"], kv)
    return eng.kv4_attention(state["q"], kv, case["ctx"], T=case["T"], own_pos0=case["ctx"] if case["own_rows"] else None,
                             visible=state.get("visible"))


def _run_plain(state):
    case, dt = state["case"], _dtype(state["case"])
    out = []
    if case["op"] != "attend":
        at, n = case["pos0"], case["rows"]
        for name, x in (("kbuf", state.get("k")), ("vbuf", state.get("v"))):
            codes, byte = _split(state[name], case)
            if case["op"] == "store":
                codes[:, at:at + n], byte[:, at:at + n] = _quantise(x.transpose(0, 1))
            out.append(_dequantise(codes[:, at:at + n], byte[:, at:at + n]).transpose(0, 1).to(dt))
        return tuple(out)
    # attention: the keys the rows may see, as float32
    n_kv, hd, C, S, T = case["n_kv"], case["hd"], case["ctx"], case["S"], case["T"]
    R = S * T
    n_own = R if case["own_rows"] else 0
    k, v = (_dequantise(c[:, :C + n_own], b[:, :C + n_own]) for c, b in (_split(state["kbuf"], case), _split(state["vbuf"], case)))
    row = torch.arange(R, device="cuda").unsqueeze(1)
    key = torch.arange(C + n_own, device="cuda").unsqueeze(0)
    limit = state["visible"].unsqueeze(1) if case["ragged"] else C
    mine = key - C
    seen = ((key < C) & (key < limit)) | ((mine >= 0) & (mine <= row) & (mine >= row - row % T))
    q = state["q"].float().unflatten(1, (n_kv, -1)).permute(1, 2, 0, 3)                 # [n_kv, group, rows, hd]
    s = (q.flatten(1, 2) @ k.transpose(1, 2)).unflatten(1, (-1, R)) / math.sqrt(hd)
    s = torch.where(seen, s, torch.full_like(s, -math.inf))
    p = torch.exp(s - s.amax(-1, keepdim=True))
    p = torch.where(seen, p, torch.zeros_like(p))
    o = (p.flatten(1, 2) @ v).unflatten(1, (-1, R)) / p.sum(-1, keepdim=True)
    o = torch.where(seen.any(1).view(1, 1, R, 1), o, torch.zeros_like(o))
    return o.permute(2, 0, 1, 3).flatten(1, 2).to(dt)


def work(case):
    n_kv, hd = case["n_kv"], case["hd"]
    esz = 4 if case["dtype"] == "fp32" else 2
    plain, packed = 2 * n_kv * hd * esz, 2 * n_kv * hd * 9 // 16       # bytes of a position's keys and values
    if case["op"] == "store":        # rows in, cache written, and read for the rows out
        return {"bytes": case["rows"] * (2 * plain + 2 * packed), "flops": 0}
    if case["op"] == "read":
        return {"bytes": case["rows"] * (plain + packed), "flops": 0}
    R, T, C = case["S"] * case["T"], case["T"], case["ctx"]
    n_own = R if case["own_rows"] else 0
    pairs = R * C * (3 / 8 if case["ragged"] else 1) + (case["S"] * T * (T + 1) / 2 if n_own else 0)
    return {"bytes": (C + n_own) * packed + 2 * R * case["n_q"] * hd * esz, "flops": 4 * hd * case["n_q"] * pairs}


# ------------------------------------------------------------------ the definition in 64 bits

def _scale64(b):
    """Scale bytes -> float64: three mantissa bits under five exponent bits."""
    e, m = (b >> 3).astype(np.int64), (b & 7).astype(np.float64)
    s = np.where(e == 0, m * 2.0 ** -17, (8.0 + m) * np.exp2(e.astype(np.float64) - 18.0))
    return np.where(b > 0xF7, np.nan, s)


def _stored64(x):
    """float64 rows -> the values the cache holds for them."""
    blocks = x.reshape(x.shape[:-1] + (x.shape[-1] // BLOCK, BLOCK))
    amax = np.abs(blocks).max(-1)
    grid = _scale64(np.arange(TOP_SCALE + 1))
    s = grid[np.minimum(np.searchsorted(grid, amax / 7.0, side="left"), TOP_SCALE)][..., None]
    c = np.clip(np.rint(np.divide(blocks, s, out=np.zeros_like(blocks), where=s > 0)), -7, 7)
    return (c * s).reshape(x.shape)


def _held64(buf, case, lo, hi):
    """Positions [lo, hi) of a cache array as float64 [n_kv, hi - lo, hd] on the GPU."""
    n, cap, hd = case["n_kv"], case["capacity"], case["hd"]
    half = n * cap * hd // 2
    codes = buf[:half].reshape(n, cap, hd // 2)[:, lo:hi].cpu().numpy()
    scale = _scale64(buf[half:].reshape(n, cap, hd // BLOCK)[:, lo:hi].cpu().numpy())
    c = np.empty(codes.shape[:-1] + (hd,), dtype=np.float64)
    c[..., 0::2], c[..., 1::2] = codes & 15, codes >> 4
    return torch.from_numpy((c - 8.0) * np.repeat(scale, BLOCK, axis=-1)).cuda()


def exact(case, seed):
    d = _inputs(case, seed)
    if case["op"] == "store":
        return tuple(torch.from_numpy(_stored64(d[x].double().cpu().numpy())).cuda() for x in ("k", "v"))
    if case["op"] == "read":
        lo, hi = case["pos0"], case["pos0"] + case["rows"]
        return tuple(_held64(d[x], case, lo, hi).transpose(0, 1) for x in ("kbuf", "vbuf"))
    C, T, R = case["ctx"], case["T"], case["S"] * case["T"]
    k, v = (_held64(d[x], case, 0, C + (R if case["own_rows"] else 0)) for x in ("kbuf", "vbuf"))
    q, G = d["q"].double(), case["n_q"] // case["n_kv"]
    out = torch.zeros((R, case["n_q"], case["hd"]), dtype=torch.float64, device="cuda")
    limits = d["visible"].tolist() if case["ragged"] else [C] * R
    whole = T > 1 and not case["ragged"]      # rows of a state in one piece, the causal part cut by a triangle
    for s in range(case["S"]):
        for r0 in range(s * T, (s + 1) * T, T if whole else 1):
            r1 = r0 + (T if whole else 1)
            cut = limits[r0]
            at = [slice(0, cut)] + ([slice(C + s * T, C + r1)] if case["own_rows"] else [])
            kk, vv = (torch.cat([x[:, a] for a in at], 1) for x in (k, v))
            if kk.shape[1] == 0:
                continue
            for g in range(case["n_kv"]):
                w = torch.einsum("rhd,kd->hrk", q[r0:r1, g * G:(g + 1) * G], kk[g]) * case["hd"] ** -0.5
                if whole:
                    late = torch.ones((r1 - r0, kk.shape[1]), dtype=torch.bool, device="cuda").triu(cut + 1)
                    w = w.masked_fill(late, -math.inf)
                out[r0:r1, g * G:(g + 1) * G] = torch.einsum("hrk,kd->rhd", torch.softmax(w, -1), vv[g])
    return out
