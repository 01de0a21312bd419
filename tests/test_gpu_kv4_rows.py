"""Rows read from a 4-bit cache: every byte in both types."""
import numpy as np
import pytest
import torch

import kv4_ref as ref
from test_gpu_kv4 import make

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
