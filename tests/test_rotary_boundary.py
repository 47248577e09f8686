"""fbl_rotary_turns, fbl_qk_norm_rotary_* and their binding refuse what they cannot compute, before any launch (CPU).
Every call here has exactly one defect."""
import ctypes
import math

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


def lay(dt=BF16, B=2, S=8, H=4, D=64, **kw):
    return F.fbl_layout_desc(dt, B, S, H, D, **kw)


def rot(**kw):
    r = F.RotaryArgs(turns=MB * 41, positions=MB * 42, stride_batch=8, stride_token=1, dims=64, num_axes=1)
    axes = kw.pop("axes", None)
    for k, v in kw.items():
        setattr(r, k, v)
    if axes is not None:
        r.axes[:len(axes)] = axes
    return r


def norm(**kw):
    return F.HeadNormArgs(**{**dict(q_weight=MB * 43, k_weight=MB * 44, eps=1e-6), **kw})


def _ref(x):
    return ctypes.byref(x) if isinstance(x, ctypes.Structure) else x


def _call(f, base, kw):
    assert set(kw) <= set(base), kw
    return f(*(_ref(v) for v in {**base, **kw}.values()))


def fwd(**kw):
    return _call(LIB.fbl_qk_norm_rotary_fwd, dict(lq=lay(), q=at(1), lk=lay(H=2), k=at(2), rot=rot(), norm=norm(), lqo=lay(),
                                                  qo=at(3), lko=lay(H=2), ko=at(4), stream=None), kw)


def bwd(**kw):
    return _call(LIB.fbl_qk_norm_rotary_bwd,
                 dict(lgq=lay(), gq=at(1), lgk=lay(H=2), gk=at(2), lq=lay(), q=at(3), lk=lay(H=2), k=at(4), rot=rot(),
                      norm=norm(), ldq=lay(), dq=at(5), ldk=lay(H=2), dk=at(6), dqw=at(7), dkw=at(8), ws=at(9),
                      ws_bytes=1 << 20, stream=None), kw)


BAD_PLAN = [
    (dict(rot=rot(turns=None)), F.FBL_ERR_NULL), (dict(rot=rot(dims=0)), F.FBL_ERR_SHAPE),
    (dict(rot=rot(dims=-16)), F.FBL_ERR_SHAPE), (dict(rot=rot(dims=80)), F.FBL_ERR_SHAPE),
    (dict(rot=rot(dims=24)), F.FBL_ERR_UNSUPPORTED), (dict(rot=rot(num_axes=0)), F.FBL_ERR_ARG),
    (dict(rot=rot(num_axes=5)), F.FBL_ERR_ARG), (dict(rot=rot(num_axes=2, axes=[0, 1, 2])), F.FBL_ERR_ARG),
    (dict(rot=rot(num_axes=2, axes=[0] * 31 + [9])), F.FBL_ERR_ARG), (dict(rot=rot(num_axes=2, positions=None)), F.FBL_ERR_NULL),
    (dict(rot=rot(neighbours=2)), F.FBL_ERR_ARG), (dict(rot=rot(reserved=1)), F.FBL_ERR_ARG),
    (dict(rot=rot(stride_token=-1)), F.FBL_ERR_LAYOUT), (dict(rot=rot(stride_batch=-8)), F.FBL_ERR_LAYOUT),
    (dict(rot=rot(stride_axis=-8)), F.FBL_ERR_LAYOUT), (dict(rot=rot(stride_batch=1 << 60)), F.FBL_ERR_LAYOUT),
    (dict(rot=rot(turns=MB * 41 + 4)), F.FBL_ERR_ALIGN), (dict(rot=rot(positions=MB * 42 + 4)), F.FBL_ERR_ALIGN),
    (dict(norm=norm(eps=-1.0)), F.FBL_ERR_ARG), (dict(norm=norm(eps=math.nan)), F.FBL_ERR_ARG),
    (dict(norm=norm(eps=math.inf)), F.FBL_ERR_ARG), (dict(norm=norm(q_weight=MB * 43 + 1)), F.FBL_ERR_ALIGN),
    (dict(norm=norm(reserved=1)), F.FBL_ERR_ARG),
]


@pytest.mark.parametrize("kw,status", BAD_PLAN + [
    (dict(lq=None), F.FBL_ERR_NULL), (dict(q=None), F.FBL_ERR_NULL), (dict(k=None), F.FBL_ERR_NULL),
    (dict(lk=None), F.FBL_ERR_NULL), (dict(qo=None), F.FBL_ERR_NULL), (dict(ko=None), F.FBL_ERR_NULL),
    (dict(lk=None, k=None), F.FBL_ERR_NULL), (dict(rot=None, norm=None), F.FBL_ERR_ARG),
    (dict(lk=lay(F32, H=2)), F.FBL_ERR_DTYPE), (dict(lqo=lay(F32)), F.FBL_ERR_DTYPE), (dict(lk=lay(H=2, S=9)), F.FBL_ERR_SHAPE),
    (dict(lk=lay(H=2, B=3)), F.FBL_ERR_SHAPE), (dict(lk=lay(H=2, D=128)), F.FBL_ERR_SHAPE), (dict(lqo=lay(H=3)), F.FBL_ERR_SHAPE),
    (dict(lko=lay(H=4)), F.FBL_ERR_SHAPE), (dict(q=at(1, 8)), F.FBL_ERR_ALIGN), (dict(ko=at(4, 2)), F.FBL_ERR_ALIGN),
    # outputs over something: another input, an input shifted, the other output, the weights, turns and positions
    (dict(qo=at(2)), F.FBL_ERR_ARG), (dict(qo=at(1, 128)), F.FBL_ERR_ARG), (dict(ko=at(3)), F.FBL_ERR_ARG),
    (dict(qo=at(1), lqo=lay(row_stride=512)), F.FBL_ERR_ARG), (dict(ko=at(1)), F.FBL_ERR_ARG), (dict(qo=at(42)), F.FBL_ERR_ARG),
    (dict(qo=at(40)), F.FBL_ERR_ARG), (dict(ko=at(43)), F.FBL_ERR_ARG), (dict(qo=at(41)), F.FBL_ERR_ARG),
])
def test_forward_refusals(kw, status):
    assert fwd(**kw) == status


@pytest.mark.parametrize("D", [16, 48, 96, 256])
def test_head_dims(D):
    l = lay(D=D)
    r, n = rot(dims=16), norm()
    assert LIB.fbl_qk_norm_rotary_fwd(_ref(l), at(1), None, None, _ref(r), _ref(n), _ref(l), at(3), None, None, None) == \
        F.FBL_ERR_UNSUPPORTED


def test_too_many_tokens():
    l = lay(B=1 << 16, S=1 << 16, H=1, D=32)
    r = rot(dims=16)
    assert LIB.fbl_qk_norm_rotary_fwd(_ref(l), at(1), None, None, _ref(r), None, _ref(l), at(1), None, None, None) == \
        F.FBL_ERR_UNSUPPORTED


@pytest.mark.parametrize("kw,status", BAD_PLAN + [
    (dict(lgq=None), F.FBL_ERR_NULL), (dict(gq=None), F.FBL_ERR_NULL), (dict(gk=None), F.FBL_ERR_NULL), (dict(q=None), F.FBL_ERR_NULL),
    (dict(k=None), F.FBL_ERR_NULL), (dict(dk=None), F.FBL_ERR_NULL), (dict(dq=None), F.FBL_ERR_NULL),
    (dict(rot=None, norm=None), F.FBL_ERR_ARG), (dict(norm=None), F.FBL_ERR_ARG),
    (dict(lgk=None, gk=None, ldk=None, dk=None, lk=None, k=None), F.FBL_ERR_ARG),  # a key weight's gradient without keys
    (dict(lq=lay(F32)), F.FBL_ERR_DTYPE), (dict(lk=lay(H=4)), F.FBL_ERR_SHAPE), (dict(ldq=lay(H=2)), F.FBL_ERR_SHAPE),
    (dict(ws=None), F.FBL_ERR_WORKSPACE), (dict(ws_bytes=1023), F.FBL_ERR_WORKSPACE), (dict(ws=at(9, 2)), F.FBL_ERR_ALIGN),
    (dict(dqw=at(7, 1)), F.FBL_ERR_ALIGN), (dict(dq=at(3)), F.FBL_ERR_ARG), (dict(dq=at(2)), F.FBL_ERR_ARG),
    (dict(dk=at(5)), F.FBL_ERR_ARG), (dict(dqw=at(8)), F.FBL_ERR_ARG), (dict(dqw=at(1)), F.FBL_ERR_ARG),
    (dict(dkw=at(6)), F.FBL_ERR_ARG), (dict(ws=at(3)), F.FBL_ERR_ARG), (dict(ws=at(8)), F.FBL_ERR_ARG),
    (dict(dqw=at(42)), F.FBL_ERR_ARG), (dict(ws=at(41)), F.FBL_ERR_ARG), (dict(dq=at(1, 128)), F.FBL_ERR_ARG),
])
def test_backward_refusals(kw, status):
    assert bwd(**kw) == status


def test_workspace():
    n = ctypes.c_size_t(7)
    f = LIB.fbl_qk_norm_rotary_bwd_workspace
    lq, lk = lay(), lay(H=2)
    assert f(_ref(lq), _ref(lk), ctypes.byref(n)) == F.FBL_OK and n.value == 2 * 2 * 64 * 4  # 16 tokens, two a wavefront
    assert f(_ref(lq), None, ctypes.byref(n)) == F.FBL_OK
    assert f(None, None, ctypes.byref(n)) == F.FBL_ERR_NULL and f(_ref(lq), None, None) == F.FBL_ERR_NULL
    assert f(_ref(lq), _ref(lay(H=2, S=9)), ctypes.byref(n)) == F.FBL_ERR_SHAPE
    big = lay(B=1 << 10, S=1 << 15, H=32, D=128)
    assert f(_ref(big), _ref(big), ctypes.byref(n)) == F.FBL_OK and n.value == 512 * 2 * 128 * 4


def test_turns():
    f = [0.0, 2 * math.pi / 4, -2 * math.pi / 4, 1.0, 1e-30, 2 * math.pi * 3.25]
    t = fbl.rotary_turns(f, device="cpu")
    assert t.dtype == torch.int64 and t.shape == (6,)
    got = [int(x) % (1 << 64) / 2.0 ** 64 for x in t]
    want = [0.0, 0.25, 0.75, 1 / (2 * math.pi), 0.0, 0.25]
    # (the frequency itself is rounded: half a step of it, in turns)
    assert all(abs(a - b) <= 2.0 ** -53 * max(1.0, abs(x)) for a, b, x in zip(got, want, f))
    assert fbl.rotary_frequencies(8, 16.0) == [1.0, 0.5, 0.25, 0.125]
    for bad, status in (([], F.FBL_ERR_SHAPE), ([1.0, math.nan], F.FBL_ERR_ARG), ([math.inf], F.FBL_ERR_ARG)):
        with pytest.raises(fbl.FblError) as e:
            fbl.rotary_turns(bad, device="cpu")
        assert e.value.status == status
    out = (ctypes.c_uint64 * 1)()
    assert LIB.fbl_rotary_turns(None, 1, out) == F.FBL_ERR_NULL
    assert LIB.fbl_rotary_turns((ctypes.c_double * 1)(1.0), 1, None) == F.FBL_ERR_NULL


def _refused(status, f, *args, **kw):
    with pytest.raises(fbl.FblError) as e:
        f(*args, **kw)
    assert e.value.status == status, e.value


def test_binding_reads_no_plan_past_its_end():
    turns = torch.zeros(32, dtype=torch.int64)
    pos = torch.zeros(2, 8, dtype=torch.int64)
    f = lambda *a: F._rotary(*a, B=2, S=8, where="here")
    ok = f(turns, pos, None, False)
    assert ok.dims == 64 and ok.num_axes == 1 and ok.stride_batch == 8 and ok.stride_token == 1
    assert f(turns, pos[0], None, False).stride_batch == 0
    three = f(turns, pos.expand(3, 2, 8), [i % 3 for i in range(32)], True)
    assert three.num_axes == 3 and three.stride_axis == 0 and three.axes[5] == 2 and three.neighbours == 1
    assert f(None, None, None, False) is None
    for args, status in (
            ((None, pos, None, False), F.FBL_ERR_ARG), ((None, None, [0], False), F.FBL_ERR_ARG),
            ((turns.int(), pos, None, False), F.FBL_ERR_DTYPE), ((turns[None], pos, None, False), F.FBL_ERR_LAYOUT),
            ((turns[::2], pos, None, False), F.FBL_ERR_LAYOUT), ((torch.zeros(65, dtype=torch.int64), pos, None, False), F.FBL_ERR_SHAPE),
            ((turns, pos.int(), None, False), F.FBL_ERR_DTYPE), ((turns, pos[:, :7], None, False), F.FBL_ERR_SHAPE),
            ((turns, pos[:1], None, False), F.FBL_ERR_SHAPE), ((turns, pos[None, None], None, False), F.FBL_ERR_SHAPE),
            ((turns, torch.zeros(0, 2, 8, dtype=torch.int64), None, False), F.FBL_ERR_SHAPE),
            ((turns, pos.expand(3, 2, 8), None, False), F.FBL_ERR_ARG), ((turns, pos.expand(5, 2, 8), [0] * 32, False), F.FBL_ERR_ARG),
            ((turns, pos, [0] * 32, False), F.FBL_ERR_SHAPE), ((turns, pos.expand(3, 2, 8), [0] * 31, False), F.FBL_ERR_SHAPE),
            ((turns, pos.expand(3, 2, 8), [3] * 32, False), F.FBL_ERR_ARG), ((turns, pos.expand(3, 2, 8), [-1] * 32, False), F.FBL_ERR_ARG),
            ((turns, None, [0] * 32, False), F.FBL_ERR_SHAPE)):
        _refused(status, f, *args)
    w = torch.ones(64)
    g = lambda *a: F._head_norm(*a, D=64, dtype=torch.float32, where="here")
    assert g(None, None, None) is None and g(w, None, 1e-6).k_weight is None
    for args, status in (((w, None, None), F.FBL_ERR_ARG), ((w[:32], None, 1e-6), F.FBL_ERR_SHAPE),
                         ((w.double(), None, 1e-6), F.FBL_ERR_DTYPE), ((None, torch.ones(128)[::2], 1e-6), F.FBL_ERR_LAYOUT)):
        _refused(status, g, *args)


def test_binding_refuses_host_tensors():
    q, t = torch.zeros(1, 4, 64), torch.zeros(16, dtype=torch.int64)
    _refused(F.FBL_ERR_ARG, fbl.qk_norm_rotary_fwd, q, None, 2, 0, turns=t)
    _refused(F.FBL_ERR_ARG, fbl.qk_norm_rotary_bwd, q, None, None, None, 2, 0, turns=t)
    _refused(F.FBL_ERR_NULL, fbl.qk_norm_rotary_bwd, q, None, None, None, 2, 0, turns=t, eps=1e-6)
    _refused(F.FBL_ERR_ARG, ag.attention_packed, torch.zeros(1, 4, 6 * 32), 2, 2, turns=t)
    _refused(F.FBL_ERR_SHAPE, ag.attention_packed, torch.zeros(1, 4, 100), 2, 2, 0.1, turns=t)


def test_a_position_alone_is_refused():
    """positions without a dimension name no tokens."""
    turns = fbl.rotary_turns(fbl.rotary_frequencies(64), device="cpu")
    with pytest.raises(fbl.FblError) as e:
        F._rotary(turns, torch.tensor(3), None, False, 1, 1, "here")
    assert e.value.status == F.FBL_ERR_SHAPE
