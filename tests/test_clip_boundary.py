"""fbl_grad_norm, fbl_grad_clip, fbl_clip_grad_norm and their binding refuse what they cannot compute, before any
launch (CPU)."""
import ctypes
import math

import pytest
import torch

import paper_2607_21624_amd as fbl
from paper_2607_21624_amd import autograd as ag
from paper_2607_21624_amd import fbl as F

LIB = F.LIB
MB = 1 << 20
BF16, F32 = F.FBL_BF16, F.FBL_F32


def at(i, off=0):
    return MB * (i + 1) + off


def lst(*changes):
    """Three tensors, the changes on the first."""
    g = (F.Grad * 3)()
    for i in range(3):
        g[i].p, g[i].out, g[i].n, g[i].dtype = at(i), at(i), 100, F32 if i == 1 else BF16
    for name, v in changes:
        setattr(g[0], name, v)
    return g


def both(n=3, g=None, limit=1.0, norm=at(8), ws=at(9), ws_bytes=1 << 20):
    return LIB.fbl_clip_grad_norm(n, lst() if g is None else g, limit, norm, ws, ws_bytes, None)


def norm_of(n=3, g=None, norm=at(8), ws=at(9), ws_bytes=1 << 20):
    return LIB.fbl_grad_norm(n, lst() if g is None else g, norm, ws, ws_bytes, None)


def clip(n=3, g=None, norm=at(8), limit=1.0):
    return LIB.fbl_grad_clip(n, lst() if g is None else g, norm, limit, None)


@pytest.mark.parametrize("f", [both, norm_of, clip])
@pytest.mark.parametrize("kw,status", [
    (dict(n=0), F.FBL_ERR_SHAPE), (dict(n=-1), F.FBL_ERR_SHAPE), (dict(n=1 << 31), F.FBL_ERR_SHAPE),
    (dict(norm=None), F.FBL_ERR_NULL), (dict(norm=at(8, 2)), F.FBL_ERR_ALIGN), (dict(g=lst(("p", None))), F.FBL_ERR_NULL),
    (dict(g=lst(("dtype", 2))), F.FBL_ERR_DTYPE), (dict(g=lst(("n", -1))), F.FBL_ERR_SHAPE),
    (dict(g=lst(("n", 1 << 45))), F.FBL_ERR_UNSUPPORTED), (dict(g=lst(("n", 1 << 62))), F.FBL_ERR_UNSUPPORTED),
    (dict(g=lst(("n", (1 << 43) + 1))), F.FBL_ERR_UNSUPPORTED),  # its chunks would not count to an int
    (dict(g=lst(("p", at(0, 1)), ("out", at(0, 1)))), F.FBL_ERR_ALIGN), (dict(g=lst(("reserved", 1))), F.FBL_ERR_ARG),
    # a tensor twice, into another, over the norm
    (dict(g=lst(("p", at(1)), ("out", at(1)))), F.FBL_ERR_ARG), (dict(g=lst(("n", MB))), F.FBL_ERR_ARG),
    (dict(norm=at(2, 100)), F.FBL_ERR_ARG),
])
def test_refusals(f, kw, status):
    assert f(**kw) == status


@pytest.mark.parametrize("f", [both, norm_of])
def test_workspace_refusals(f):
    n = ctypes.c_size_t()
    assert LIB.fbl_grad_norm_workspace(3, ctypes.byref(n)) == F.FBL_OK and n.value == 1024 * 8
    assert f(ws=None) == F.FBL_ERR_WORKSPACE and f(ws_bytes=n.value - 1) == F.FBL_ERR_WORKSPACE
    assert f(ws=at(9, 4)) == F.FBL_ERR_ALIGN and f(ws=at(1)) == F.FBL_ERR_ARG and f(ws=at(8) - 8) == F.FBL_ERR_ARG
    assert LIB.fbl_grad_norm_workspace(113, ctypes.byref(n)) == F.FBL_OK and n.value == 2 * 1024 * 8
    assert LIB.fbl_grad_norm_workspace(0, ctypes.byref(n)) == F.FBL_ERR_SHAPE
    assert LIB.fbl_grad_norm_workspace(3, None) == F.FBL_ERR_NULL


@pytest.mark.parametrize("f", [both, clip])
def test_output_refusals(f):
    for g, status in ((lst(("out", None)), F.FBL_ERR_NULL), (lst(("out", at(5, 1))), F.FBL_ERR_ALIGN),
                      (lst(("out", at(0, 2))), F.FBL_ERR_ARG), (lst(("out", at(1))), F.FBL_ERR_ARG),
                      (lst(("out", at(8))), F.FBL_ERR_ARG)):
        assert f(g=g) == status
    for limit in (-1.0, math.nan):
        assert f(limit=limit) == F.FBL_ERR_ARG


def _refused(status, f, *args, **kw):
    with pytest.raises(fbl.FblError) as e:
        f(*args, **kw)
    assert e.value.status == status, e.value


def test_binding_refusals():
    t = torch.zeros(4, 6)
    for f in (lambda g, **kw: fbl.grad_norm(g), lambda g, **kw: fbl.clip_grad_norm(g, 1.0, **kw),
              lambda g, **kw: fbl.clip_grads(g, torch.zeros(()), 1.0, **kw)):
        _refused(F.FBL_ERR_SHAPE, f, [])
        _refused(F.FBL_ERR_ARG, f, [t])       # not on a GPU
        _refused(F.FBL_ERR_ARG, f, [t, 3.0])  # no tensor
    _refused(F.FBL_ERR_SHAPE, fbl.clip_grad_norm, [t], 1.0, out=[t, t])
    _refused(F.FBL_ERR_NULL, fbl.clip_grads, [t], None, 1.0)  # whose norm?
    p = torch.zeros(3, requires_grad=True)
    _refused(F.FBL_ERR_SHAPE, ag.clip_grad_norm_, [p], 1.0)  # no gradient at all
    _refused(F.FBL_ERR_SHAPE, fbl.grad_norm_workspace, [])


def test_dense():
    t = torch.zeros(4, 6, 5)
    for yes in (t, t.permute(2, 0, 1), t[1], t.transpose(0, 2), t[1, :4], torch.zeros(()), t[:0], t[2:3]):
        assert F._dense(yes)
    assert F._dense(torch.zeros(3, 1, 4).permute(1, 2, 0)) and F._dense(torch.zeros(0, 7)[:, ::2])
    for no in (t[:, ::2], t[..., :4], t[:, :3], torch.zeros(5).expand(3, 5)):
        assert not F._dense(no)
