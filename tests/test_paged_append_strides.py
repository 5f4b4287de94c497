"""lg_paged_append takes contiguous rows where no strides are given, and only there: strides of zero are refused, all three of them too, on the
host.  No GPU."""
import ctypes as C

import pytest

from paper_2410_01485_b200 import binding as lg, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return lg.load_library()


@pytest.mark.parametrize("T", [1, 4])
@pytest.mark.parametrize("strides", [(0, 0, 0), (0, 0, 128), (0, 1024, 0), (2048, 0, 0), (2048, 1024, 0), (2048, 0, 128)])
def test_zero_strides(lib, T, strides):
    p = lg.paged_params(2, 8, 2, 128, 64, 256, page_tokens=32, num_pages=40)
    assert lib.lg_paged_append(C.byref(p), 256, 512, 256, 512, 256, 256, 256, (C.c_int64 * 3)(*strides), T, 256, None, None) == -1


def test_binding_refuses_an_expanded_row(lib, monkeypatch):
    """A row broadcast over sequences, heads and tokens has three strides of zero."""
    import torch
    monkeypatch.setattr(lg, "_check_device", lambda *tensors: None)          # (nothing reaches a device)
    monkeypatch.setattr(lg, "_stream", lambda: None)
    p = lg.paged_params(2, 8, 2, 128, 64, 256, page_tokens=32, num_pages=40)
    pools = [torch.zeros(40, 2, 32, 128, dtype=torch.uint8) for _ in "kv"]
    scales = [torch.ones(40, 2) for _ in "kv"]
    table, n = torch.zeros(2, 10, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    row = torch.zeros(128, dtype=torch.bfloat16).expand(2, 2, 4, 128)
    assert row.stride() == (0, 0, 0, 1)
    with pytest.raises(lg.LgError) as e:
        lg.lg_paged_append(p, *pools, *scales, table, row, row, n)
    assert e.value.code == -1
