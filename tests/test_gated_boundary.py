"""fbl_gated_* and their binding refuse what they cannot compute, before any launch (CPU).  Every call here has
exactly one defect."""
import ctypes

import pytest
import torch

import paper_2607_21624_amd as fbl
from paper_2607_21624_amd import autograd as ag
from paper_2607_21624_amd import fbl as F

LIB = F.LIB
MB = 1 << 20  # made-up device addresses, never dereferenced
BF16, F32 = F.FBL_BF16, F.FBL_F32


def at(i, off=0):
    return ctypes.c_void_p(MB * (i + 1) + off)


def _call(f, base, kw):
    assert set(kw) <= set(base), kw
    return f(*{**base, **kw}.values())


def fwd(**kw):
    return _call(LIB.fbl_gated_fwd, dict(dt=BF16, act=F.FBL_ACT_SILU, M=4, K=64, F=32, x=at(1), ldx=64, w=at(2), ldw=64,
                                         b=at(3), h=at(4), ldh=32, f=at(5), ldf=64, tile=-1, ws=None, ws_bytes=0, stream=None), kw)


def bwd(**kw):
    return _call(LIB.fbl_gated_bwd, dict(dt=BF16, M=4, F=32, N=64, dy=at(1), lddy=64, wd=at(2), ldwd=64,
                                         f=at(3), ldf=64, dz=at(4), lddz=64, db=at(5), tile=-1, ws=at(6), ws_bytes=1 << 20,
                                         stream=None), kw)


COMMON = [(dict(dt=2), F.FBL_ERR_DTYPE), (dict(M=0), F.FBL_ERR_SHAPE), (dict(M=-1), F.FBL_ERR_SHAPE),
          (dict(F=0), F.FBL_ERR_SHAPE), (dict(tile=21), F.FBL_ERR_ARG), (dict(tile=-2), F.FBL_ERR_ARG)]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(act=5), F.FBL_ERR_ARG), (dict(K=0), F.FBL_ERR_SHAPE), (dict(K=(1 << 26) + 8, ldx=(1 << 26) + 8), F.FBL_ERR_UNSUPPORTED),
    (dict(F=(1 << 25) + 8, ldw=(1 << 26) + 16, ldh=(1 << 25) + 8, ldf=(1 << 26) + 16, M=1), F.FBL_ERR_UNSUPPORTED),
    (dict(M=1 << 24), F.FBL_ERR_UNSUPPORTED),  # factors of 2 GiB
    (dict(x=None), F.FBL_ERR_NULL), (dict(w=None), F.FBL_ERR_NULL), (dict(h=None), F.FBL_ERR_NULL),
    (dict(ldx=56), F.FBL_ERR_LAYOUT), (dict(ldw=56), F.FBL_ERR_LAYOUT), (dict(ldh=24), F.FBL_ERR_LAYOUT),
    (dict(ldf=56), F.FBL_ERR_LAYOUT), (dict(ldw=68), F.FBL_ERR_ALIGN), (dict(x=at(1, 8)), F.FBL_ERR_ALIGN),
    (dict(b=at(3, 8)), F.FBL_ERR_ALIGN), (dict(K=60), F.FBL_ERR_UNSUPPORTED), (dict(F=28), F.FBL_ERR_UNSUPPORTED),
    (dict(h=at(1)), F.FBL_ERR_ARG), (dict(h=at(2)), F.FBL_ERR_ARG), (dict(h=at(3)), F.FBL_ERR_ARG), (dict(f=at(4)), F.FBL_ERR_ARG),
    (dict(f=at(1)), F.FBL_ERR_ARG), (dict(dt=F32, tile=0), F.FBL_ERR_ARG), (dict(dt=F32, x=at(1, 2)), F.FBL_ERR_ALIGN),
    # a contraction that is shared
    (dict(K=4096, ldx=4096, ws=at(9), ws_bytes=1023), F.FBL_ERR_WORKSPACE),
    (dict(K=4096, ldx=4096, ws=at(9, 8), ws_bytes=1 << 30), F.FBL_ERR_ALIGN),
    (dict(K=4096, ldx=4096, ws=at(4), ws_bytes=1 << 30), F.FBL_ERR_ARG),
])
def test_forward_refusals(kw, status):
    assert fwd(**kw) == status


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(N=0), F.FBL_ERR_SHAPE), (dict(dy=None), F.FBL_ERR_NULL), (dict(wd=None), F.FBL_ERR_NULL), (dict(f=None), F.FBL_ERR_NULL),
    (dict(dz=None), F.FBL_ERR_NULL), (dict(lddy=56), F.FBL_ERR_LAYOUT), (dict(ldwd=32), F.FBL_ERR_LAYOUT),
    (dict(ldf=32), F.FBL_ERR_LAYOUT), (dict(lddz=56), F.FBL_ERR_LAYOUT), (dict(dz=at(4, 2)), F.FBL_ERR_ALIGN),
    (dict(db=at(5, 1)), F.FBL_ERR_ALIGN), (dict(N=60), F.FBL_ERR_UNSUPPORTED), (dict(F=28), F.FBL_ERR_UNSUPPORTED),
    (dict(M=1 << 24), F.FBL_ERR_UNSUPPORTED), (dict(ws=None), F.FBL_ERR_WORKSPACE), (dict(ws_bytes=512), F.FBL_ERR_WORKSPACE),
    (dict(ws=at(6, 8)), F.FBL_ERR_ALIGN), (dict(dz=at(3)), F.FBL_ERR_ARG), (dict(dz=at(1)), F.FBL_ERR_ARG),
    (dict(db=at(4)), F.FBL_ERR_ARG), (dict(ws=at(3)), F.FBL_ERR_ARG), (dict(ws=at(5)), F.FBL_ERR_ARG),
    (dict(dt=F32, tile=3), F.FBL_ERR_ARG),
])
def test_backward_refusals(kw, status):
    assert bwd(**kw) == status


def test_workspaces_are_functions_of_the_shape():
    n = ctypes.c_size_t(7)
    f, b = LIB.fbl_gated_fwd_workspace, LIB.fbl_gated_bwd_workspace
    assert f(BF16, 4096, 2048, 8192, ctypes.byref(n)) == F.FBL_OK and n.value == 0
    assert f(BF16, 1, 4096, 4096, ctypes.byref(n)) == F.FBL_OK and n.value > 0 and n.value % (2 * 4096 * 4) == 0
    assert b(BF16, 4096, 8192, 2048, ctypes.byref(n)) == F.FBL_OK and n.value == (4096 // 32 + 4) * 2 * 8192 * 4
    for g in (f, b):
        assert g(BF16, 4, 64, 32, None) == F.FBL_ERR_NULL and g(7, 4, 64, 32, ctypes.byref(n)) == F.FBL_ERR_DTYPE
        assert g(BF16, 0, 64, 32, ctypes.byref(n)) == F.FBL_ERR_SHAPE


def test_workspace_holds_every_tile_s_sums():
    """The rows of partial sums of any tile of the table, for any number of tokens, fit what the workspace keeps."""
    tiles = fbl.gemm_tiles()
    for M in (1, 31, 32, 33, 127, 128, 129, 255, 257, 1000, 4097):
        assert all(-(-M // t["bm"]) * t["wm"] <= M // 32 + 4 for t in tiles.values()), M


@pytest.mark.parametrize("F_", [8, 1032, 8192])
def test_workspace_of_shared_contractions_holds_every_tile_s_sums(F_):
    """A tile that the caller names does not share the contraction: behind the planes that AUTO would use the workspace has
    room for that tile's rows of partial sums, and for the one row a token that the shared path writes."""
    n = ctypes.c_size_t()
    tiles = fbl.gemm_tiles()
    rows = lambda M: max(max(-(-M // t["bm"]) * t["wm"] for t in tiles.values()), M)
    for N in (64, 2048, 2056, 4096, 8192, 16384):
        for M in range(1, 129):
            # (the forward of a linear layer of the same extents keeps its planes alone)
            assert LIB.fbl_linear_fwd_workspace(BF16, M, N, F_, ctypes.byref(n)) == F.FBL_OK
            planes = (n.value + 255) // 256 * 256
            if not planes:
                continue
            assert LIB.fbl_gated_bwd_workspace(BF16, M, F_, N, ctypes.byref(n)) == F.FBL_OK
            assert n.value - planes >= rows(M) * 2 * F_ * 4, (M, F_, N)


def _refused(status, f, *args, **kw):
    with pytest.raises(fbl.FblError) as e:
        f(*args, **kw)
    assert e.value.status == status, e.value


def test_binding_refusals():
    x, w, z = torch.zeros(4, 64), torch.zeros(64, 64), torch.zeros(4, 64)
    _refused(F.FBL_ERR_ARG, fbl.gated_fwd, x, w)  # not on a GPU
    _refused(F.FBL_ERR_ARG, fbl.gated_bwd, x, w, z)
    _refused(F.FBL_ERR_SHAPE, F._gated_width, torch.zeros(64, 63), "here")
    _refused(F.FBL_ERR_SHAPE, fbl.gated_fwd_workspace, x, torch.zeros(64, 63))
    _refused(F.FBL_ERR_SHAPE, ag.gated_mlp, x, w, None, torch.zeros(32, 64), None, residual=torch.zeros(3, 64))
