"""Pins of the float64 oracle of per-head norms with rotation, the gated feed-forward part and clipping (CPU): central
differences, torch in float64, closed forms."""
import decimal
import math

import numpy as np
import pytest
import torch

from oracle import gated_block as G
from test_oracle_train import ACTS, _diff


@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("dims,eps", [(8, 1e-5), (4, 1e-5), (8, None), (0, 1e-5)])
def test_norm_rotary_differences(neighbours, dims, eps):
    rng = np.random.default_rng(dims)
    x, dy, w = rng.normal(size=(2, 3, 2, 8)), rng.normal(size=(2, 3, 2, 8)), rng.normal(1, 0.2, 8)
    pos = rng.integers(-50, 50, (2, 3))
    angle = G.angles(pos, [10.0 ** -j for j in range(dims // 2)]) if dims else None
    w = w if eps is not None else None
    dx, dw = G.qk_norm_rotary_bwd(dy, x, angle, neighbours, w, eps)
    f = lambda: float((G.qk_norm_rotary_fwd(x, angle, neighbours, w, eps) * dy).sum())
    _diff(f, x, dx, n=40)
    if w is not None:
        _diff(f, w, dw, n=8)
    else:
        assert dw is None


def test_rotation_closed_forms():
    x = np.random.default_rng(0).normal(size=(1, 4, 3, 16))
    # position 0 and a whole turn leave x; lengths of pairs stay; angles add
    assert np.array_equal(G.rotate(x, np.zeros((1, 4, 8))), x)
    a = np.random.default_rng(1).normal(size=(1, 4, 6))
    for nb in (False, True):
        y = G.rotate(x, a, nb)
        assert np.array_equal(y[..., 12:], x[..., 12:])
        i, j = G._pairs(16, 12, nb)
        assert np.allclose(y[..., i] ** 2 + y[..., j] ** 2, x[..., i] ** 2 + x[..., j] ** 2)
        assert np.allclose(G.rotate(y, a, nb), G.rotate(x, 2 * a, nb))
        assert np.allclose(G.rotate(x, np.full((1, 4, 6), math.pi / 2), nb)[..., i], -x[..., j])
    # a score depends on the difference of positions alone
    q, k = x[:, :1], x[:, 1:2]
    f = [1.0, 0.1, 0.01, 0.001]
    at = lambda m, n: (G.rotate(q, G.angles([[m]], f)) * G.rotate(k, G.angles([[n]], f))).sum(-1)
    assert np.allclose(at(5, 2), at(105, 102)) and not np.allclose(at(5, 2), at(5, 3))


def test_angles_of_axes():
    pos = np.arange(2 * 3).reshape(3, 1, 2) * 7
    a = G.angles(pos, [1.0, 0.5, 0.25], [2, 0, 1])
    assert np.allclose(np.cos(a[0, 1]), np.cos([35 * 1.0, 7 * 0.5, 21 * 0.25]))


def test_angles_of_far_positions():
    """Ordinary frequencies at positions where the product has many whole turns, against 100 decimal digits: within two roundings
    of a float64 of at most pi."""
    turn = decimal.Decimal("6.28318530717958647692528676655900576839433879875021164194988918461563281257241799725606965")
    far = [0, 1, -1, 4097, -(1 << 20), 10 ** 9 + 7, (1 << 31) - 1, -(1 << 31), 1 << 40, -(10 ** 15) - 3, (1 << 63) - 1, -(1 << 63)]
    freq = [1.0, 1e4 ** -0.25, 5e5 ** -0.5, 1e4 ** (-62 / 64), 0.7]
    a = G.angles(np.array([far]), freq)
    with decimal.localcontext() as c:
        c.prec = 100
        for i, n in enumerate(far):
            for j, f in enumerate(freq):
                want = decimal.Decimal(n) * decimal.Decimal(f)
                want -= turn * (want / turn).to_integral_value(decimal.ROUND_HALF_EVEN)
                assert abs(decimal.Decimal(a[0, i, j]) - want) <= 2 * decimal.Decimal(2) ** -52, (n, f)


@pytest.mark.parametrize("kind", ACTS)
def test_gated_differences(kind):
    rng = np.random.default_rng(3)
    x, w, b, dh = (rng.normal(size=s) for s in ((4, 5), (5, 12), (12,), (4, 6)))
    h, z = G.gated_fwd(x, w, b, kind)
    dz = G.gated_bwd(dh, G.gated_factors(z, kind))
    f = lambda: float((G.gated_fwd(x, w, b, kind)[0] * dh).sum())
    for a, g in ((x, dz @ w.T), (w, x.T @ dz), (b, dz.sum(0))):
        _diff(f, a, g)
    fn = {"none": lambda t: t, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
          "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}[kind]
    t = torch.from_numpy(z)
    assert np.allclose(h, (fn(t[:, :6]) * t[:, 6:]).numpy(), rtol=0, atol=1e-12)


def test_clip():
    grads = [np.full((3, 4), 2.0), np.full(4, -3.0)]
    assert math.isclose(G.grad_norm(grads), math.sqrt(12 * 4 + 4 * 9))
    n = torch.nn.utils.get_total_norm([torch.from_numpy(g) for g in grads])
    assert math.isclose(G.grad_norm(grads), float(n))
    p = [torch.zeros(g.shape, dtype=torch.float64).requires_grad_(True) for g in grads]
    for t, g in zip(p, grads):
        t.grad = torch.from_numpy(g.copy())
    torch.nn.utils.clip_grad_norm_(p, 2.5)
    assert np.allclose(p[0].grad.numpy(), grads[0] * G.clip_scale(G.grad_norm(grads), 2.5), rtol=1e-12)
    assert G.clip_scale(1.0, 2.0) == 1.0


def test_kept_factors():
    """Within 2^13 of the largest of eight 2^-11 of the value, else 2^-24 of the largest; any exponent of fp32."""
    rng = np.random.default_rng(5)
    for scale in (1.0, 2.0 ** -126, 2.0 ** -140, 2.0 ** 120, 1e-30, 3e4):
        v = np.float32(rng.standard_normal((40, 64)) * 10.0 ** rng.uniform(-6, 0, (40, 64)) * scale)
        got = G.kept_factors(G.keep_factors(v))
        top = np.repeat(np.abs(v).reshape(40, -1, 8).max(-1), 8, axis=-1)
        assert np.all(np.abs(got - v) <= np.maximum(2.0 ** -11 * np.abs(v.astype(np.float64)), 2.0 ** -24 * top))
    v = np.float32([[0] * 8 + [1, -1, 0.5, 65504, 2.0 ** -126, 0, 0, -3e38], [1, 2, 4, 8, 16, 32, 64, 128] * 2])
    got = G.kept_factors(G.keep_factors(v))
    assert np.all(got[0, :8] == 0) and np.all(got[1] == v[1]) and got[0, 12] == 0
    assert np.all(np.isinf(G.kept_factors(np.full((1, 8), 0xffff, np.uint16))))
