"""The most rows of the adapters' calls: what every launch takes is accepted by the workspace queries, more is refused by
the queries and the calls alike, before anything touches a device."""
import ctypes
import os

import pytest

from paper_2609_40093_amd import _lib

D = ctypes.c_void_p(1 << 20)  # never dereferenced
MOST = 2 ** 30 - 2 ** 21      # EP_ADAPTER_MAX_ROWS


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2609_40093_amd import build
        build.build()
    return _lib.load()


def answers(lib, rows, R):
    """The statuses of both queries and, where they are to refuse, of both calls."""
    n, m = ctypes.c_size_t(), ctypes.c_size_t()
    got = [lib.ep_adapter_product_workspace_bytes(rows, 1, R, 8, 8, 0, 0, ctypes.byref(n)),
           lib.ep_adapter_product_grad_workspace_bytes(rows, 1, R, 8, 8, 0, 0, 0, 7, ctypes.byref(m))]
    if rows * -(-R // 64) > MOST:
        got += [lib.ep_adapter_product(D, rows, None, None, 1, R, D, D, None, None, 8, 8, None, 0, None, None, None, D, D, 1 << 50,
                                       None),
                lib.ep_adapter_product_grad(D, rows, None, None, 1, R, D, D, None, None, 8, 8, D, 0, None, D, D, D, D, D, 1 << 50,
                                            None)]
    return got


@pytest.mark.parametrize("R,columns", [(8, 1), (64, 1), (72, 2), (136, 3), (256, 4)])
def test_most_rows(lib, R, columns):
    most = MOST // columns
    assert answers(lib, most, R) == [_lib.EP_OK] * 2
    for rows in (most + 1, 2 * most, 2 ** 31 - 1):
        assert answers(lib, rows, R) == [_lib.EP_ERR_INVALID_ARG] * 4, rows
        assert b"rows" in lib.ep_last_error()
