"""The layer operators' refusals of what no grid holds, on the host."""
import ctypes as C

import pytest

from paper_2109_12497_b200 import binding as B
from paper_2109_12497_b200 import build as uq_build

P = 0x10000


@pytest.fixture(scope="module")
def lib():
    uq_build.build()
    return B.lib()


def test_binary32_columns_of_more_tiles_than_a_grid_has_blocks(lib):
    """2^31 tiles of 32 x 128, of fewer than 2^31 tiles of 64 x 64: binary32 columns go by the former."""
    rows, cols = 1 << 30, 64 * 127
    qt = B.uq_mx(cols, rows, 1 << 29, P, P)
    q = B.uq_mx(rows, cols, 4096, P, P)
    for along_rows in (None, C.byref(q)):
        assert lib.uq_mx_quantize(P, rows, cols, cols, B.UQ_F32, 0, 0, along_rows, C.byref(qt), None, None) == B.UQ_ERR_UNSUPPORTED
