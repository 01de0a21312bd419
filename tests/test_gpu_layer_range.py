"""clasp_layer_forward near the end of the 32-bit positions: refused before a launch."""
import ctypes as C

import pytest
import torch

import datagen
import paper_2505_24196_b200 as clasp
from util import Pair

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("flags", [0, clasp.FLAG_KV4, clasp.FLAG_MULTI_KERNEL])
def test_positions_whose_end_passes_32_bits_are_refused(flags):
    cfg = datagen.CONFIGS["small"]
    p = Pair(cfg, 96, 32, max_M=2, flags=flags)
    eng = p.engine
    kv = (clasp.KV4Cache if flags & clasp.FLAG_KV4 else clasp.KVCache)(p.ccfg)
    x = torch.zeros((8, cfg.d_model), device="cuda")
    out = torch.zeros_like(x)
    layer = clasp.ClaspKvLayer(kv.array[1].k, kv.array[1].v)
    call = lambda T, ctx, pos, write: eng.lib.clasp_layer_forward(eng.handle, 1, x.data_ptr(), cfg.d_model, 1, T, ctx, pos,
                                                                  C.byref(layer), write, out.data_ptr(), cfg.d_model)
    n0 = eng.launch_count()
    for write in (0, 1):
        for T in (1, 2, 8):
            for pos in (2 ** 31 - 1, 2 ** 31 - T, 96 - T + 1, 96):
                assert call(T, 5, pos, write) == -3, (T, pos, write)
    assert eng.launch_count() == n0
    assert call(8, 88, 88, 1) == 0 and eng.device_status() == 0
