"""Host-side argument handling of the 4-bit cache's calls, without a device."""
import pytest
import torch

import paper_2505_24196_b200 as clasp


def unbound(dtype=torch.bfloat16):
    """A Clasp without a context: what _head_rows looks at."""
    eng = object.__new__(clasp.Clasp)
    eng._hd, eng.dtype, eng._index, eng.workspace = 128, dtype, -1, torch.empty(0, dtype=torch.uint8)
    return eng


def test_stride_of_rows():
    eng = unbound()
    rows = lambda n, stride, h: torch.zeros((8, stride), dtype=torch.bfloat16)[:, :h * 128].unflatten(1, (h, 128))[:n]
    assert eng._head_rows(rows(5, 2 * 128, 2), 2, "k") == 256
    assert eng._head_rows(rows(5, 3 * 128, 2), 2, "k") == 384
    # nothing steps over the stride of a single row, whatever it is
    for stride in (256, 257, 384, 1001):
        assert rows(1, stride, 2).stride(0) == stride
        assert eng._head_rows(rows(1, stride, 2), 2, "k") == 256
    assert eng._head_rows(rows(1, 256, 2).as_strided((1, 2, 128), (0, 128, 1)), 2, "k") == 256
    assert eng._head_rows(rows(0, 384, 2), 2, "k") == 256
    # rows that lie on one another are handed on as they are: the library refuses them
    assert eng._head_rows(rows(1, 256, 2).expand(4, 2, 128), 2, "k") == 0


def test_rows_that_are_refused():
    eng = unbound()
    ok = torch.zeros((3, 2, 128), dtype=torch.bfloat16)
    assert eng._head_rows(ok, 2, "k") == 256
    for bad in (ok.float(), ok[..., :64], ok[:, :1], ok[0], ok.transpose(0, 1), ok.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises(ValueError):
            eng._head_rows(bad, 2, "k")
