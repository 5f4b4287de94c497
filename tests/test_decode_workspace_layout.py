"""What a decode workspace holds in front of its records lies where no call's sizes move it: from one batch to a larger one the workspace
grows by records alone.  No GPU."""
import ctypes as C

import pytest

from paper_2410_01485_b200 import binding, build


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def check_growth(size, D):
    batches = [1, 4, 8, 9, 16, 40, 41, 300]
    sizes = [size(B, D) for B in batches]
    record = 8 * (D + 2) * 4                                     # 8 heads: O and (maximum, sum); 8 kv heads of one group each
    for (b0, s0), (b1, s1) in zip(zip(batches, sizes), zip(batches[1:], sizes[1:])):
        assert s1 - s0 == -(-(320 + 8 * b1) * record // 256) * 256 - -(-(320 + 8 * b0) * record // 256) * 256


@pytest.mark.parametrize("D", [64, 128])
def test_paged(lib, D):
    check_growth(lambda B, d: lib.lg_paged_decode_workspace_bytes(C.byref(
        binding.paged_params(B, 64, 8, d, 128, 4096, page_tokens=64, num_pages=100))), D)


@pytest.mark.parametrize("D", [64, 128])
def test_ring(lib, D):
    check_growth(lambda B, d: lib.lg_sparse_decode_workspace_bytes(C.byref(binding.decode_params(B, 64, 8, d, 128, 4096))), D)
