"""The entry points of layer norm, linear layers and the losses refuse what they cannot
compute, before any launch (CPU).  Every call here has exactly one defect."""
import ctypes

import pytest
import torch

import paper_2607_21624_amd as fbl
from paper_2607_21624_amd import fbl as F

LIB = F.LIB
FAKE = 1 << 20  # made-up device addresses, 1 MiB apart, never dereferenced
BF16, F32 = F.FBL_BF16, F.FBL_F32


def at(i, off=0):
    return ctypes.c_void_p(FAKE * (i + 1) + off)


def _merge(base, kw):
    assert set(kw) <= set(base), kw
    return list({**base, **kw}.values())


def norm_fwd(**kw):
    return LIB.fbl_layer_norm_fwd(*_merge(dict(dt=BF16, M=4, N=64, x=at(1), ldx=64, w=at(2), b=at(3), eps=1e-5, y=at(4),
                                               ldy=64, mean=at(5), rstd=at(6), stream=None), kw))


def norm_bwd(**kw):
    return LIB.fbl_layer_norm_bwd(*_merge(dict(dt=BF16, M=4, N=64, dy=at(1), lddy=64, x=at(2), ldx=64, w=at(3),
                                               mean=at(4), rstd=at(5), dx=at(6), lddx=64, dw=at(7), db=at(8), ws=at(9),
                                               ws_bytes=1 << 20, stream=None), kw))


@pytest.mark.parametrize("kw,status", [
    (dict(dt=2), F.FBL_ERR_DTYPE), (dict(M=0), F.FBL_ERR_SHAPE), (dict(N=-1), F.FBL_ERR_SHAPE),
    (dict(M=1 << 31), F.FBL_ERR_SHAPE), (dict(N=16385, ldx=16385, ldy=16385), F.FBL_ERR_UNSUPPORTED),
    (dict(x=None), F.FBL_ERR_NULL), (dict(y=None), F.FBL_ERR_NULL), (dict(mean=None), F.FBL_ERR_NULL),
    (dict(rstd=None), F.FBL_ERR_NULL), (dict(ldx=63), F.FBL_ERR_LAYOUT), (dict(ldy=63), F.FBL_ERR_LAYOUT),
    (dict(ldx=1 << 31), F.FBL_ERR_LAYOUT), (dict(eps=-1e-5), F.FBL_ERR_ARG), (dict(eps=float("nan")), F.FBL_ERR_ARG),
    (dict(x=at(1, 1)), F.FBL_ERR_ALIGN), (dict(y=at(4, 1)), F.FBL_ERR_ALIGN), (dict(mean=at(5, 2)), F.FBL_ERR_ALIGN),
    (dict(y=at(1)), F.FBL_ERR_ARG), (dict(y=at(1, 64 * 2)), F.FBL_ERR_ARG), (dict(mean=at(2)), F.FBL_ERR_ARG),
    (dict(rstd=at(5)), F.FBL_ERR_ARG), (dict(M=(1 << 31) - 1, ldx=(1 << 31) - 1), F.FBL_ERR_SHAPE),
    # columns 32 .. 95 of rows of 96 against columns 0 .. 63
    (dict(ldx=96, ldy=96, y=at(1, 32 * 2)), F.FBL_ERR_ARG),
])
def test_layer_norm_fwd_refusals(kw, status):
    assert norm_fwd(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=-1), F.FBL_ERR_DTYPE), (dict(M=-4), F.FBL_ERR_SHAPE), (dict(N=1 << 20, lddy=1 << 20, ldx=1 << 20, lddx=1 << 20),
                                                                   F.FBL_ERR_UNSUPPORTED),
    (dict(dy=None), F.FBL_ERR_NULL), (dict(x=None), F.FBL_ERR_NULL), (dict(mean=None), F.FBL_ERR_NULL),
    (dict(rstd=None), F.FBL_ERR_NULL), (dict(dx=None), F.FBL_ERR_NULL), (dict(lddy=0), F.FBL_ERR_LAYOUT),
    (dict(lddx=60), F.FBL_ERR_LAYOUT), (dict(ws=None), F.FBL_ERR_WORKSPACE), (dict(ws_bytes=511), F.FBL_ERR_WORKSPACE),
    (dict(ws=at(9, 2)), F.FBL_ERR_ALIGN), (dict(rstd=at(5, 1)), F.FBL_ERR_ALIGN), (dict(dx=at(1)), F.FBL_ERR_ARG),
    (dict(dw=at(3)), F.FBL_ERR_ARG), (dict(db=at(7)), F.FBL_ERR_ARG), (dict(ws=at(6)), F.FBL_ERR_ARG),
])
def test_layer_norm_bwd_refusals(kw, status):
    assert norm_bwd(**kw) == status


def test_layer_norm_workspace():
    n = ctypes.c_size_t(7)
    f = LIB.fbl_layer_norm_bwd_workspace
    assert f(BF16, 4, 64, ctypes.byref(n)) == F.FBL_OK and n.value == 1 * 2 * 64 * 4  # 4 rows: one workgroup's sums
    assert f(BF16, 4, 64, None) == F.FBL_ERR_NULL
    assert f(9, 4, 64, ctypes.byref(n)) == F.FBL_ERR_DTYPE
    assert f(F32, 0, 64, ctypes.byref(n)) == F.FBL_ERR_SHAPE
    assert f(F32, 4, 16385, ctypes.byref(n)) == F.FBL_ERR_UNSUPPORTED
    assert f(BF16, 1 << 30, 16384, ctypes.byref(n)) == F.FBL_OK and n.value == 256 * 2 * 16384 * 4


def test_layer_norm_binding_refuses_host_tensors():
    x = torch.zeros(4, 64)
    for f in (lambda: fbl.layer_norm_fwd(x), lambda: fbl.layer_norm_bwd(x, x, x[:, 0], x[:, 0])):
        with pytest.raises(fbl.FblError) as e:
            f()
        assert e.value.status == F.FBL_ERR_ARG


# ----------------------------------------------------------------- linear layers
def lin_fwd(**kw):
    return LIB.fbl_linear_fwd(*_merge(dict(dt=BF16, act=2, M=8, K=64, N=64, x=at(1), ldx=64, w=at(2), ldw=64, bias=at(3),
                                           res=at(4), ldr=64, y=at(5), ldy=64, z=at(6), ldz=64, tile=-1, ws=None, ws_bytes=0, stream=None), kw))


def lin_bwd(**kw):
    return LIB.fbl_linear_bwd(*_merge(dict(dt=BF16, act=2, M=8, K=64, N=64, dy=at(1), lddy=64, x=at(2), ldx=64, w=at(3),
                                           ldw=64, z=at(4), ldz=64, xact=3, xz=at(5), ldxz=64, dx=at(6), lddx=64, dxbias=None,
                                           dw=at(7), lddw=64, dbias=at(8), ws=at(9), ws_bytes=1 << 19, stream=None), kw))


@pytest.mark.parametrize("kw,status", [
    (dict(dt=5), F.FBL_ERR_DTYPE), (dict(act=5), F.FBL_ERR_ARG), (dict(M=0), F.FBL_ERR_SHAPE), (dict(K=0), F.FBL_ERR_SHAPE),
    (dict(N=1 << 31), F.FBL_ERR_SHAPE), (dict(x=None), F.FBL_ERR_NULL), (dict(w=None), F.FBL_ERR_NULL),
    (dict(y=None), F.FBL_ERR_NULL), (dict(ldx=56), F.FBL_ERR_LAYOUT), (dict(ldr=0), F.FBL_ERR_LAYOUT),
    (dict(ldz=63), F.FBL_ERR_LAYOUT), (dict(ldw=68), F.FBL_ERR_ALIGN), (dict(x=at(1, 8)), F.FBL_ERR_ALIGN),
    (dict(bias=at(3, 2)), F.FBL_ERR_ALIGN), (dict(z=at(6, 4)), F.FBL_ERR_ALIGN), (dict(K=60), F.FBL_ERR_UNSUPPORTED),
    (dict(N=62), F.FBL_ERR_UNSUPPORTED), (dict(tile=21), F.FBL_ERR_ARG), (dict(tile=-2), F.FBL_ERR_ARG),
    (dict(dt=F32, tile=0), F.FBL_ERR_ARG), (dict(dt=F32, x=at(1, 2)), F.FBL_ERR_ALIGN),
    (dict(y=at(1)), F.FBL_ERR_ARG), (dict(y=at(4)), F.FBL_ERR_ARG), (dict(z=at(5)), F.FBL_ERR_ARG),
    (dict(z=at(3)), F.FBL_ERR_ARG), (dict(M=1 << 25), F.FBL_ERR_UNSUPPORTED), (dict(ldx=1 << 28), F.FBL_ERR_UNSUPPORTED),
])
def test_linear_fwd_refusals(kw, status):
    assert lin_fwd(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dt=5), F.FBL_ERR_DTYPE), (dict(act=5), F.FBL_ERR_ARG), (dict(xact=9), F.FBL_ERR_ARG), (dict(M=-1), F.FBL_ERR_SHAPE),
    (dict(dy=None), F.FBL_ERR_NULL), (dict(x=None), F.FBL_ERR_NULL), (dict(w=None), F.FBL_ERR_NULL),
    (dict(z=None), F.FBL_ERR_NULL), (dict(xz=None), F.FBL_ERR_NULL), (dict(ws=None), F.FBL_ERR_WORKSPACE),
    (dict(ws_bytes=1000), F.FBL_ERR_WORKSPACE), (dict(ws=at(9, 8)), F.FBL_ERR_ALIGN), (dict(lddx=32), F.FBL_ERR_LAYOUT),
    (dict(dbias=at(8, 1)), F.FBL_ERR_ALIGN), (dict(N=68, lddy=72, ldw=72, ldz=72, lddw=72), F.FBL_ERR_UNSUPPORTED),
    (dict(dx=at(1)), F.FBL_ERR_ARG), (dict(dw=at(6)), F.FBL_ERR_ARG), (dict(dbias=at(7)), F.FBL_ERR_ARG),
    (dict(ws=at(5)), F.FBL_ERR_ARG), (dict(dx=at(5)), F.FBL_ERR_ARG), (dict(dxbias=at(10, 1)), F.FBL_ERR_ALIGN),
    (dict(dxbias=at(6)), F.FBL_ERR_ARG), (dict(dxbias=at(8)), F.FBL_ERR_ARG), (dict(dxbias=at(3)), F.FBL_ERR_ARG),
    (dict(dxbias=at(10), dx=None), F.FBL_ERR_NULL), (dict(dxbias=at(9)), F.FBL_ERR_ARG),
    (dict(act=0, dbias=None, dxbias=at(10), ws=None), F.FBL_ERR_WORKSPACE),
])
def test_linear_bwd_refusals(kw, status):
    assert lin_bwd(**kw) == status


def test_linear_workspace_and_binding():
    n = ctypes.c_size_t()
    f = LIB.fbl_linear_bwd_workspace
    assert f(BF16, 8, 64, 64, ctypes.byref(n)) == F.FBL_OK and n.value >= 8 * 64 * 2 + 64 * 4
    assert f(BF16, 8, 64, 64, None) == F.FBL_ERR_NULL
    assert f(7, 8, 64, 64, ctypes.byref(n)) == F.FBL_ERR_DTYPE
    assert f(F32, 8, 0, 64, ctypes.byref(n)) == F.FBL_ERR_SHAPE
    assert f(F32, (1 << 31) - 1, 64, (1 << 31) - 1, ctypes.byref(n)) == F.FBL_ERR_UNSUPPORTED
    x = torch.zeros(4, 64)
    for call in (lambda: fbl.linear_fwd(x, x.t()), lambda: fbl.linear_bwd(x, x, x)):
        with pytest.raises(fbl.FblError) as e:
            call()
        assert e.value.status == F.FBL_ERR_ARG


# ------------------------------------------------------- losses of a linear head
def ce_fwd(**kw):
    return LIB.fbl_linear_ce_fwd(*_merge(dict(dt=BF16, order=1, M=8, K=64, V=100, x=at(1), ldx=64, w=at(2), ldw=64, labels=at(3),
                                              ignore=-100, loss=at(4), lse=at(5), total=at(6), mean=at(7), ws=at(8),
                                              ws_bytes=1 << 19, stream=None), kw))


def ce_bwd(**kw):
    return LIB.fbl_linear_ce_bwd(*_merge(dict(dt=BF16, order=1, M=8, K=64, V=100, dloss=at(1), stride=0, total=at(2), x=at(3),
                                              ldx=64, w=at(4), ldw=64, labels=at(5), ignore=-100, lse=at(6), dx=at(7), lddx=64,
                                              dw=at(8), lddw=64, ws=at(9), ws_bytes=1 << 19, stream=None), kw))


def kd_fwd(**kw):
    return LIB.fbl_linear_kd_fwd(*_merge(dict(dt=BF16, order=0, M=8, K=64, V=104, top=4, x=at(1), ldx=64, w=at(2), ldw=104,
                                              index=at(3), ldi=4, ldt=F32, logits=at(4), ldl=4, T=2.0, prob=at(5), loss=at(6),
                                              lse=at(7), total=at(8), mean=at(9), ws=at(10), ws_bytes=1 << 19, stream=None), kw))


def kd_bwd(**kw):
    return LIB.fbl_linear_kd_bwd(*_merge(dict(dt=BF16, order=0, M=8, K=64, V=104, top=4, dloss=at(1), stride=1, total=None,
                                              x=at(2), ldx=64, w=at(3), ldw=104, index=at(4), ldi=4, T=2.0, prob=at(5), lse=at(6),
                                              dx=at(7), lddx=64, dw=at(8), lddw=104, ws=at(9), ws_bytes=1 << 19, stream=None),
                                         kw))


COMMON = [
    (dict(dt=3), F.FBL_ERR_DTYPE), (dict(order=2), F.FBL_ERR_ARG), (dict(M=0), F.FBL_ERR_SHAPE), (dict(K=-8), F.FBL_ERR_SHAPE),
    (dict(V=1 << 31), F.FBL_ERR_SHAPE), (dict(K=60), F.FBL_ERR_UNSUPPORTED), (dict(M=1 << 24), F.FBL_ERR_UNSUPPORTED),
    (dict(x=None), F.FBL_ERR_NULL), (dict(w=None), F.FBL_ERR_NULL), (dict(lse=None), F.FBL_ERR_NULL),
    (dict(ldx=56), F.FBL_ERR_LAYOUT), (dict(ldw=56), F.FBL_ERR_LAYOUT), (dict(ldx=68), F.FBL_ERR_ALIGN),
    (dict(w=at(2, 4)), F.FBL_ERR_ALIGN), (dict(lse=at(5, 2)), F.FBL_ERR_ALIGN), (dict(ws=None), F.FBL_ERR_WORKSPACE),
    (dict(ws_bytes=64), F.FBL_ERR_WORKSPACE), (dict(ws=at(8, 8)), F.FBL_ERR_ALIGN),
    (dict(dt=F32, x=at(1, 2), ldx=64), F.FBL_ERR_ALIGN),
]


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(labels=None), F.FBL_ERR_NULL), (dict(loss=None), F.FBL_ERR_NULL), (dict(total=None), F.FBL_ERR_NULL),  # mean needs total
    (dict(labels=at(3, 4)), F.FBL_ERR_ALIGN), (dict(order=0, V=100, ldw=104), F.FBL_ERR_UNSUPPORTED),
    (dict(loss=at(1)), F.FBL_ERR_ARG), (dict(lse=at(4)), F.FBL_ERR_ARG), (dict(ws=at(2)), F.FBL_ERR_ARG),
    (dict(mean=at(6, 4)), F.FBL_ERR_ARG), (dict(total=at(8)), F.FBL_ERR_ARG), (dict(loss=at(3)), F.FBL_ERR_ARG),
])
def test_linear_ce_fwd_refusals(kw, status):
    assert ce_fwd(**kw) == status


@pytest.mark.parametrize("kw,status", COMMON + [
    (dict(dloss=None), F.FBL_ERR_NULL), (dict(labels=None), F.FBL_ERR_NULL), (dict(stride=-1), F.FBL_ERR_LAYOUT),
    (dict(lddx=0), F.FBL_ERR_LAYOUT), (dict(lddw=63), F.FBL_ERR_LAYOUT), (dict(dx=at(7, 8)), F.FBL_ERR_ALIGN),
    (dict(dw=at(8, 2)), F.FBL_ERR_ALIGN), (dict(dloss=at(1, 1)), F.FBL_ERR_ALIGN), (dict(dx=at(3)), F.FBL_ERR_ARG),
    (dict(dw=at(4)), F.FBL_ERR_ARG), (dict(dw=at(7)), F.FBL_ERR_ARG), (dict(ws=at(6)), F.FBL_ERR_ARG),
])
def test_linear_ce_bwd_refusals(kw, status):
    assert ce_bwd(**kw) == status


@pytest.mark.parametrize("kw,status", [(k, s) for k, s in COMMON if "ldw" not in k and "lse" not in k and "ws" not in k] + [
    (dict(top=0), F.FBL_ERR_SHAPE), (dict(top=1025, ldi=1025, ldl=1025), F.FBL_ERR_UNSUPPORTED), (dict(T=0.0), F.FBL_ERR_ARG),
    (dict(T=-1.0), F.FBL_ERR_ARG), (dict(T=float("inf")), F.FBL_ERR_ARG), (dict(T=float("nan")), F.FBL_ERR_ARG),
    (dict(index=None), F.FBL_ERR_NULL), (dict(logits=None), F.FBL_ERR_NULL), (dict(prob=None), F.FBL_ERR_NULL),
    (dict(ldt=4), F.FBL_ERR_DTYPE), (dict(ldi=3), F.FBL_ERR_LAYOUT), (dict(ldl=3), F.FBL_ERR_LAYOUT), (dict(ldw=103), F.FBL_ERR_LAYOUT),
    (dict(ldw=108), F.FBL_ERR_ALIGN), (dict(V=100), F.FBL_ERR_UNSUPPORTED), (dict(prob=at(3)), F.FBL_ERR_ARG),
    (dict(prob=at(6)), F.FBL_ERR_ARG), (dict(index=at(3, 4)), F.FBL_ERR_ALIGN), (dict(ws=at(4)), F.FBL_ERR_ARG),
])
def test_linear_kd_fwd_refusals(kw, status):
    assert kd_fwd(**kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(top=-1), F.FBL_ERR_SHAPE), (dict(T=0.0), F.FBL_ERR_ARG), (dict(index=None), F.FBL_ERR_NULL), (dict(prob=None), F.FBL_ERR_NULL),
    (dict(lse=None), F.FBL_ERR_NULL), (dict(ldi=2), F.FBL_ERR_LAYOUT), (dict(prob=at(5, 2)), F.FBL_ERR_ALIGN),
    (dict(dx=at(5)), F.FBL_ERR_ARG), (dict(dw=at(3)), F.FBL_ERR_ARG), (dict(ws=at(2)), F.FBL_ERR_ARG),
    (dict(ws_bytes=100), F.FBL_ERR_WORKSPACE), (dict(lddw=96), F.FBL_ERR_LAYOUT),
])
def test_linear_kd_bwd_refusals(kw, status):
    assert kd_bwd(**kw) == status


def test_linear_loss_workspace():
    n = ctypes.c_size_t()
    f = lambda dt=BF16, order=1, M=4096, K=1024, V=50257, top=1, ldw=1024: LIB.fbl_linear_loss_workspace(
        dt, order, M, K, V, top, ldw, ctypes.byref(n))
    assert f() == F.FBL_OK
    # never the logits of 50257 entries, let alone in fp32: pieces of 128 MiB, 16 MiB of sums and lists
    assert n.value < 4096 * 50257 * 2 / 2
    assert f(V=16) == F.FBL_OK and n.value < 1 << 20
    assert LIB.fbl_linear_loss_workspace(BF16, 1, 8, 64, 64, 1, 64, None) == F.FBL_ERR_NULL
    assert f(dt=9) == F.FBL_ERR_DTYPE and f(order=3) == F.FBL_ERR_ARG and f(V=0) == F.FBL_ERR_SHAPE
    assert f(ldw=1000) == F.FBL_ERR_LAYOUT and f(ldw=1028) == F.FBL_ERR_ALIGN and f(top=1025) == F.FBL_ERR_UNSUPPORTED
    # [K, V] rows beyond a span are refused, a table of any size is not
    assert f(order=0, K=8192, V=262144, ldw=262144) == F.FBL_ERR_UNSUPPORTED
    assert f(order=1, K=8192, V=262144, ldw=8192) == F.FBL_OK


def test_losses_binding_refuses_host_tensors_and_layouts():
    x, w, lab = torch.zeros(4, 64), torch.zeros(64, 100), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: fbl.linear_ce_fwd(x, w, lab), lambda: fbl.linear_kd_fwd(x, w, lab[:, None], x[:, :1]),
                 lambda: fbl.linear_ce_bwd(x[0, 0], x, w, lab, x[:, 0]),
                 lambda: fbl.linear_kd_bwd(x[0, 0], x, w, lab[:, None], x[:, :1], x[:, 0])):
        with pytest.raises(fbl.FblError) as e:
            call()
        assert e.value.status == F.FBL_ERR_ARG
    head = F._head
    assert head(w, x, "") == (0, 100) and head(torch.zeros(100, 64).t(), x, "") == (1, 64)
    assert head(torch.zeros(64, 120)[:, :100], x, "") == (0, 120) and head(torch.zeros(100, 80)[:, :64].t(), x, "") == (1, 80)
    with pytest.raises(fbl.FblError) as e:
        head(torch.zeros(64, 200)[:, ::2], x, "")
    assert e.value.status == F.FBL_ERR_LAYOUT
    with pytest.raises(fbl.FblError) as e:
        head(torch.zeros(1, 100).expand(64, 100), x, "")  # one row for all
    assert e.value.status == F.FBL_ERR_LAYOUT


def test_linear_width_limits():
    n = ctypes.c_size_t()
    f = LIB.fbl_linear_bwd_workspace
    assert f(F32, 1, 8, (1 << 26) + 1, ctypes.byref(n)) == F.FBL_ERR_UNSUPPORTED
    assert f(F32, 1, (1 << 26) + 1, 8, ctypes.byref(n)) == F.FBL_ERR_UNSUPPORTED
    assert f(F32, 1, 8, 1 << 26, ctypes.byref(n)) == F.FBL_OK
