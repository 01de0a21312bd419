"""Host-only checks of the 4-bit cache's entry points and of the plain form its GPU tests compare with."""
import ctypes as C

import numpy as np

import datagen
import kv4_ref as ref
import paper_2505_24196_b200 as clasp


def config(flags=clasp.FLAG_KV4, **kw):
    cfg = clasp.make_config(datagen.CONFIGS["8b"], max_ctx=1000, max_rows=64, max_M=16, flags=flags)
    for k, v in kw.items():
        setattr(cfg, k, v)
    return cfg


def test_bytes_of_a_cache():
    lib = clasp.load_library()
    assert lib.clasp_kv4_bytes(config()) == 8 * 1000 * (64 + 8)
    assert lib.clasp_kv4_bytes(config(head_dim=64)) == 8 * 1000 * (32 + 4)
    assert lib.clasp_kv4_bytes(config(max_ctx=1 << 30)) == (1 << 30) * 8 * 72        # past 32 bits
    for bad in (config(flags=0), config(head_dim=96), config(max_ctx=(1 << 30) + 1), config(n_kv_heads=5)):
        assert lib.clasp_kv4_bytes(bad) == 0
    assert lib.clasp_kv4_bytes(None) == 0
    assert lib.clasp_workspace_bytes(config(max_ctx=(1 << 30) + 1)) == 0
    # no buffers of the persistent kernel, partial results of at most 64 rows
    assert 0 < lib.clasp_workspace_bytes(config(max_rows=2048)) < lib.clasp_workspace_bytes(config(flags=0, max_rows=2048))


def test_calls_without_a_context_are_refused():
    lib = clasp.load_library()
    layer = clasp.ClaspKvLayer(16, 16)
    assert lib.clasp_kv4_write(None, 16, 1024, 16, 1024, 1, 0, C.byref(layer)) == -1
    assert lib.clasp_kv4_read(None, C.byref(layer), 0, 1, 16, 1024, 16, 1024) == -1
    assert lib.clasp_kv4_attention(None, 16, 4096, 1, 1, 1, -1, None, C.byref(layer), 16, 4096) == -1


def test_plain_form_of_the_format():
    """The reference the GPU tests use: scales are the half-precision numbers of their bits, the scale is the smallest that
    holds the block, codes are nearest, what is stored is exact in bf16."""
    half = (np.arange(256, dtype=np.uint16) << 7).view(np.float16).astype(np.float64)
    ok = np.arange(256) < 0xF8
    np.testing.assert_array_equal(ref.TABLE[ok], half[ok])
    assert ref.TABLE[ref.TOP] == 896.0 and np.isnan(ref.TABLE[ref.BAD])
    rng = np.random.default_rng(0)
    x = rng.standard_normal((500, 64)) * np.exp2(rng.integers(-20, 14, (500, 4))).repeat(16, -1)
    x[3, :16] = 0.0
    x[4, 5] = np.inf
    x[5, 20] = np.nan
    c, b = ref.quantise(x)
    v = ref.values(c, b)
    assert c.min() >= 1 and c.max() <= 15
    assert (v[3, :16] == 0).all() and np.isnan(v[4, :16]).all() and np.isnan(v[5, 16:32]).all()
    good = np.isfinite(v).reshape(500, 4, 16).all(-1)
    s = ref.TABLE[b]
    amax = np.abs(np.where(np.isfinite(x), x, 0)).reshape(500, 4, 16).max(-1)
    top = b == ref.TOP
    assert (7 * s >= amax)[good & ~top].all()
    assert ((b == 0) | (7 * ref.TABLE[np.maximum(b, 1) - 1] < amax))[good].all()
    err = np.abs(x - v).reshape(500, 4, 16).max(-1)
    assert (err <= s / 2)[good & ~top].all()
    bits = np.ascontiguousarray(v[good.repeat(16, -1).reshape(500, 64)].astype(np.float32)).view(np.uint32)
    assert ((bits & 0xFFFF) == 0).all()


def test_plain_attention_of_nothing_and_of_one_key():
    q, k, v = np.ones((2, 4, 64)), np.ones((3, 2, 64)), np.arange(3.0)[:, None, None] * np.ones((3, 2, 64))
    seen = np.array([[False, False, False], [False, True, False]])
    out, _, _ = ref.attention(q, k, v, seen)
    assert (out[0] == 0).all() and (out[1] == 1.0).all()
    m = ref.seen_mask(4, 2, 3, True, [-1, 0, 2, 9])
    assert m[:, :3].sum(1).tolist() == [0, 0, 2, 3] and m[:, 3:].tolist() == [[1, 0, 0, 0], [1, 1, 0, 0], [0, 0, 1, 0], [0, 0, 1, 1]]
