"""The native call path of the rotation with its norms, gated layers and clipping against the general one: the same
results bit for bit, and None -- the general path -- for every call that is not a plain one."""
import pytest
import torch

import paper_2607_21624_amd as pkg
from ops_util import DTYPES, note
from paper_2607_21624_amd import fbl
from test_gpu_fastcall_ops import _both, _t

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_rotation(monkeypatch, dt):
    dt = DTYPES[dt]
    note(f"native rotation {dt}")
    qkv, g = _t(2, 9, 8 * 64, dt=dt), _t(2, 9, 6 * 64, dt=dt)
    q, k, gq, gk = qkv[..., :256], qkv[..., 256:384], g[..., :256], g[..., 256:]
    w = _t(64, dt=dt)
    turns = pkg.rotary_turns(pkg.rotary_frequencies(32))
    pos = torch.randint(0, 1000, (3, 2, 9), device="cuda")
    axes = tuple(i % 3 for i in range(16))
    for kw in (dict(turns=turns), dict(turns=turns, positions=pos[0], neighbours=True), dict(turns=turns, positions=pos[0, 0]),
               dict(turns=turns, positions=pos, axes=axes, eps=1e-6), dict(eps=1e-5, q_weight=w), dict(turns=turns, positions=pos[:1]),
               dict(turns=turns, eps=1e-6, q_weight=w, k_weight=w)):
        _both(monkeypatch, lambda: pkg.qk_norm_rotary_fwd(q, k, 4, 2, **kw))
        _both(monkeypatch, lambda: pkg.qk_norm_rotary_fwd(q, None, 4, 0, **kw))
        _both(monkeypatch, lambda: pkg.qk_norm_rotary_bwd(gq, gk, q, k, 4, 2, **kw))
        _both(monkeypatch, lambda: pkg.qk_norm_rotary_bwd(gq, gk, q, k, 4, 2, need_weights=False, **kw))
        _both(monkeypatch, lambda: pkg.qk_norm_rotary_bwd(gq, None, q, None, 4, 0, **kw))
    out = torch.empty(2, 9, 512, dtype=dt, device="cuda")
    _both(monkeypatch, lambda: pkg.qk_norm_rotary_fwd(q, k, 4, 2, turns=turns, q_out=out[..., :256], k_out=out[..., 256:384]))
    _both(monkeypatch, lambda: pkg.qk_norm_rotary_bwd(gq, gk, None, None, 4, 2, turns=turns, dq=out[..., :256], dk=out[..., 256:384]))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_gated(monkeypatch, dt):
    dt = DTYPES[dt]
    g = lambda *s, **k: _t(*s, dt=dt, **k)
    note(f"native gated {dt}")
    for M in (1, 50, 300):
        x, w, b, wd, dy = g(M, 264), g(264, 144), g(144), g(72, 136), g(M, 136)
        f = torch.empty(M, 144, dtype=dt, device="cuda")
        for act in pkg.ACTIVATIONS:
            _both(monkeypatch, lambda: pkg.gated_fwd(x, w, b, act, factors=f))
            _both(monkeypatch, lambda: pkg.gated_bwd(dy, wd, f))
            _both(monkeypatch, lambda: pkg.gated_bwd(dy, wd, f, need_bias=False, dz=torch.empty_like(f)))
        _both(monkeypatch, lambda: pkg.gated_fwd(x, w, out=torch.empty(M, 72, dtype=dt, device="cuda")))
    _both(monkeypatch, lambda: pkg.gated_fwd(g(4, 4096, scale=0) + 1, g(4096, 144, scale=0) + 1))  # shared contraction


def test_clipping(monkeypatch):
    note("native clipping")
    grads = [_t(30, 20), _t(7, dt=torch.float32), _t(64, 3).t(), _t(0, 4)]
    out = [torch.empty_like(t) for t in grads]
    _both(monkeypatch, lambda: pkg.grad_norm(grads))
    _both(monkeypatch, lambda: pkg.grad_norm(tuple(grads), norm=torch.empty((), device="cuda")))
    _both(monkeypatch, lambda: pkg.clip_grad_norm(grads, 1.0, out=out))
    a = [t.clone() for t in out]
    _both(monkeypatch, lambda: pkg.clip_grad_norm(grads, 1.0, out=tuple(out)))
    assert all(torch.equal(x, y) for x, y in zip(a, out))
    own = [t.clone() for t in grads]
    assert fbl._FAST.clip_grad_norm(own, 1.0, None, None, None, None) is not None
    assert all(torch.equal(x, y) for x, y in zip(own, out))


def test_other_calls_go_the_general_way():
    q, t, w = _t(2, 9, 256), pkg.rotary_turns(pkg.rotary_frequencies(32)), _t(64)
    fast, side = fbl._FAST, torch.cuda.Stream()
    rot = lambda *a, q=q, stream=None: fast.qk_norm_rotary_fwd(q, None, 4, 0, *a, None, None, stream)
    assert rot(t, None, None, False, None, None, None) is not None
    pos = torch.zeros(2, 9, dtype=torch.int64, device="cuda")
    for a in ((t.int(), None, None, False, None, None, None), (t, pos.int(), None, False, None, None, None),
              (t, pos[:, :8], None, False, None, None, None), (t, pos, (0,) * 16, False, None, None, None),
              (t, pos.expand(3, 2, 9), None, False, None, None, None), (t, pos.expand(3, 2, 9), (3,) * 16, False, None, None, None),
              (t, pos.expand(3, 2, 9), [0] * 16, False, None, None, None), (None, pos, None, False, None, None, None),
              (None, None, None, False, None, None, None), (t, None, None, 0, None, None, None), (t, None, None, False, w, None, None),
              (t, None, None, False, w[:32], None, 1e-6), (t, None, None, False, None, None, 1)):
        assert rot(*a) is None, a
    assert rot(t, None, None, False, None, None, None, stream=side) is None
    assert rot(t, None, None, False, None, None, None, q=q[..., :250]) is None
    bwd = lambda g, k: fast.qk_norm_rotary_bwd(g, None, q, k, 4, 0, t, None, None, False, None, None, 1e-6, None, None, None, None,
                                               None, None, True)
    assert bwd(q, None) is not None and bwd(q, q) is None and bwd(q[:, :8], None) is None
    x, w1 = _t(4, 64), _t(64, 32)
    assert fast.gated_fwd(x, w1, None, "silu", None, None, -1, None, None) is not None
    assert fast.gated_fwd(x, w1, None, "swish", None, None, -1, None, None) is None
    assert fast.gated_fwd(x, _t(64, 31), None, "silu", None, None, -1, None, None) is None
    assert fast.gated_fwd(x, w1, None, "silu", None, None, -1, None, side) is None
    assert fast.gated_bwd(x, _t(16, 64), _t(4, 30), None, None, -1, None, None, False) is None
    assert fast.gated_bwd(x, _t(16, 64), _t(4, 32), None, None, -1, None, None, False) is not None
    g = [_t(4, 6), _t(3)]
    for a in (g + [None], [], [g[0], g[0]], [g[0][:, :3]], [g[0].half()], iter(g), [g[0].cpu()]):
        assert fast.clip_grad_norm(a, 1.0, None, None, None, None) is None
    assert fast.clip_grad_norm(g, 1, None, None, None, None) is None and fast.clip_grad_norm(g, -1.0, None, None, None, None) is None
    assert fast.clip_grad_norm(g, 1.0, g[:1], None, None, None) is None
    assert fast.clip_grad_norm(g, 1.0, [g[1], g[0]], None, None, None) is None
    assert fast.grad_norm(g, torch.zeros(2, device="cuda"), None, None) is None and fast.grad_norm(g, None, None, side) is None
