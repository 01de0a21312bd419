"""Rows written to and read from a 4-bit cache: every byte in both types, addresses and strides that are multiples of 16 bytes
and of no more, single rows with any stride."""
import numpy as np
import pytest
import torch

import kv4_ref as ref
import paper_2505_24196_b200 as clasp
from test_gpu_kv4 import dt, make, rows, special_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("hd", [64, 128])
def test_read_every_code_and_scale_in_both_types(dtype, hd):
    """(c - 8) s for all 16 codes under all 256 scale bytes.  0xF8 is an infinite scale: infinities, and NaN for the code 8."""
    n_kv, cap, per = 2, 64, hd // 16
    eng, kv = make((4, n_kv, hd), cap, dtype=dtype)
    b = np.arange(n_kv * cap * per).reshape(n_kv, cap, per) & 255
    for buf in (kv.k, kv.v):
        a = np.zeros(buf.shape[1], dtype=np.uint8)
        codes, scales = ref.parts(a, n_kv, cap, hd)
        pair = np.arange(8, dtype=np.uint8) * 2
        codes[:] = np.tile(pair + ((pair + 1) << 4), per)
        scales[:] = b
        buf[0].copy_(torch.from_numpy(a))
    half = (np.arange(256, dtype=np.uint16) << 7).view(np.float16).astype(np.float64)
    with np.errstate(invalid="ignore"):
        want = ((np.arange(16) - 8.0) * half[b][..., None]).reshape(n_kv, cap, hd).transpose(1, 0, 2)
    for got in eng.kv4_read(0, cap, kv):
        np.testing.assert_array_equal(ref.to_np(got), want)


@pytest.mark.parametrize("heads", [(8, 2, 128), (4, 2, 64), (8, 1, 128)])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("offset,pad", [(16, 0), (0, 16), (16, 16), (32, 0), (0, 32), (48, 80)])
def test_rows_at_multiples_of_sixteen_bytes(heads, dtype, offset, pad):
    """Rows `offset` bytes behind a 32-byte border and `pad` bytes apart: written, read back and left alone around them."""
    n_q, n_kv, hd = heads
    esz = 2 if dtype == "bf16" else 4
    n, row, cap = 37, n_kv * hd, 64
    stride, start = row + pad // esz, offset // esz
    eng, kv = make(heads, cap, dtype=dtype)

    def place(fill):
        buf = torch.full((start + n * stride + 64,), fill, dtype=dt(dtype), device="cuda")
        assert buf.data_ptr() % 32 == 0
        return buf, buf[start:start + n * stride].view(n, stride)[:, :row].unflatten(1, (n_kv, hd))

    x = [special_rows(n, n_kv, hd, dtype, s) for s in (11, 23)]
    src = [place(5.0)[1] for _ in x]
    for s, t in zip(src, x):
        s.copy_(t)
    kv.k.fill_(0xA5)
    kv.v.fill_(0xA5)
    eng.kv4_write(src[0], src[1], 3, kv)
    dst = [place(9.0) for _ in x]
    eng.kv4_read(3, n, kv, k_out=dst[0][1], v_out=dst[1][1])
    torch.cuda.synchronize()
    for buf, t, (whole, got) in zip((kv.k, kv.v), x, dst):
        want = np.full(buf.shape[1], 0xA5, dtype=np.uint8)
        c, b = ref.quantise(ref.to_np(t))
        ref.pack(c, b, want, n_kv, cap, hd, 3)
        np.testing.assert_array_equal(buf[0].cpu().numpy(), want)
        np.testing.assert_array_equal(ref.to_np(got), ref.values(c, b))
        got.fill_(9.0)
        assert bool((whole == 9.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("odd", [1, 3, 7])
def test_a_single_row_has_no_stride(dtype, odd):
    """One row cut from a buffer whose rows are any number of elements apart: nothing steps over that stride."""
    heads = (8, 2, 128)
    eng, kv = make(heads, 32, dtype=dtype)

    def one(h):
        t = torch.zeros((2, h * 128 + odd), dtype=dt(dtype), device="cuda")[:, :h * 128].unflatten(1, (h, 128))[:1]
        assert t.stride(0) == h * 128 + odd
        return t

    k, v, q = one(2), one(2), one(8)
    for i, t in enumerate((k, v, q)):
        t.copy_(rows(i, tuple(t.shape), dtype))
    eng.kv4_write(k, v, 4, kv)
    back = one(2), one(2)
    eng.kv4_read(4, 1, kv, k_out=back[0], v_out=back[1])
    out = one(8)
    assert eng.kv4_attention(q, kv, 4, own_pos0=4, out=out) is out
    clean = [t.contiguous() for t in (k, v, q)]
    want = clasp.KV4Cache(eng.cfg)
    eng.kv4_write(clean[0], clean[1], 4, want)
    assert torch.equal(kv.k, want.k) and torch.equal(kv.v, want.v)
    assert all(torch.equal(a, b) for a, b in zip(back, eng.kv4_read(4, 1, kv)))
    assert torch.equal(out, eng.kv4_attention(clean[2], kv, 4, own_pos0=4))
