"""What the operators' workspaces have to hold, from their sizes (CPU)."""
import ctypes

import pytest

from paper_2607_21624_amd import fbl as F

LIB = F.LIB


def _size(f, *args):
    n = ctypes.c_size_t()
    assert f(*args, ctypes.byref(n)) == F.FBL_OK
    return n.value


@pytest.mark.parametrize("N", [4, 12, 260, 1028])
def test_rows_of_dz_are_whole_chunks(N):
    """bf16 products stage their operands by aligned 16-byte loads, dz like any other: with N % 8 == 4 its rows
    take the room of N + 4.  (K N is above the weights whose gradient workgroups share, M above the tokens of a
    shared dx: what remains is dz and sums that M does not multiply with N.)"""
    M, K = 100000, max(4096, 2 ** 20 // N // 8 * 8)
    size = lambda n: _size(LIB.fbl_linear_bwd_workspace, F.FBL_BF16, M, K, n)
    # sums over blocks of rows: at most 512 rows of N + 4 fp32, and roundings to 256 bytes
    assert size(N + 4) - size(N) <= 512 * 4 * 4 + 3 * 256
    assert size(N) >= M * (N + 4) * 2
