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


@pytest.mark.parametrize("table", [False, True])
@pytest.mark.parametrize("dt,es", [(F.FBL_BF16, 2), (F.FBL_F32, 4)])
@pytest.mark.parametrize("M", [1, 16, 100, 128, 129, 700, 4096, 8192, 16384, 32768, 65536, 131072])
@pytest.mark.parametrize("K,V", [(64, 50256), (1024, 50256), (2048, 128256), (512, 1000)])
def test_losses_workspace_is_within_its_bound(K, V, M, dt, es, table):
    """A piece of dz, sums of dX, the forward's parts and the targets' lists, as the header states them."""
    if not table and K * V * es >= 1 << 31:
        return
    for top in (1, 50):
        got = _size(LIB.fbl_linear_loss_workspace, dt, F.FBL_HEAD_VK if table else F.FBL_HEAD_KV, M, K, V, top, K if table else V)
        rows = M * es
        dz = min(rows * (V + 63), max(128 << 20, 4096 * rows) + 64 * rows, 1 << 31)
        sums = max(M * K * 4, 64 << 20)
        parts = M * 8 * (-(-V // 32) + 16)
        lists = 2 * M * top * 4 + 3 * 8 * M
        assert got <= max(dz + sums, parts) + lists + 4096
        if M >= 4096 and rows * V > 256 << 20:  # and pieces are not small
            assert got >= 32 << 20


@pytest.mark.parametrize("dt,es", [(F.FBL_BF16, 2), (F.FBL_F32, 4)])
def test_nothing_is_shared_where_the_binding_brings_no_workspace(dt, es):
    """The binding asks for a forward's workspace up to 128 tokens, and for a plain backward's up to 128 tokens or
    weights of 2^19; what the library could share beyond that it would leave alone, unnoticed.  There no size may have
    room for planes (two of them at least): a block of bias sums, dz and dx's sums are all."""
    for M in (129, 136, 200, 256, 300, 512, 1000, 4096, 8192, 100000):
        for K in (64, 512, 1032, 2048, 4096, 8192, 16384):
            for N in (64, 264, 1024, 4096, 8200, 32768):
                if M * max(K, N) * es >= 1 << 31:
                    continue
                assert _size(LIB.fbl_linear_fwd_workspace, dt, M, K, N) == 0
                if K * N > 1 << 19:
                    most = 512 * N * 4 + M * N * es + (M // 32 + 4) * K * 4 + 3 * 256
                    assert _size(LIB.fbl_linear_bwd_workspace, dt, M, K, N) <= most, (M, K, N)
