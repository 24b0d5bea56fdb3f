"""The workspace of the adapters' product keeps to what its path needs, from the smallest sizes to the longest rows and
largest ranks."""
import ctypes
import os

import pytest

from paper_2609_40093_amd import _lib


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_40093_amd import build
        build.build()
    return _lib.load()


@pytest.mark.parametrize("R", [8, 64, 256])
@pytest.mark.parametrize("K", [8, 1024, 16384, 262144])
@pytest.mark.parametrize("N", [8, 1024])
def test_parts_of_low_rank_values(lib, R, K, N):
    """Without W nothing is kept but low-rank values: two bf16 values of each rank, rounded up to whole blocks, or the parts of
    their sums, of which many rows have no more bytes than those."""
    n = ctypes.c_size_t()
    for rows in (1, 10, 100, 500, 1000, 3000, 8700, 15000, 100000):
        assert lib.ep_adapter_product_workspace_bytes(rows, 1, R, K, N, 0, 0, ctypes.byref(n)) == _lib.EP_OK
        blocks = -(-R // (32 if R <= 32 else 64)) * (32 if R <= 32 else 64)
        assert n.value <= max(64 << 20, rows * blocks * 2 * 2 + 256), (rows, n.value)
