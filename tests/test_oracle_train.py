"""Pins of the float64 oracle of layer norm, linear layers with an epilogue and the
losses of a linear head (CPU): central differences, float64 torch autograd, closed forms."""
import math

import numpy as np
import pytest
import torch

from oracle import train as T

ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _diff(f, a, g, h=1e-5, n=12, seed=0):
    """Central differences of the scalar f at n entries of `a`, against the gradient g."""
    rng = np.random.default_rng(seed)
    for i in rng.choice(a.size, size=min(n, a.size), replace=False):
        at = np.unravel_index(i, a.shape)
        keep = a[at]
        a[at] = keep + h
        up = f()
        a[at] = keep - h
        down = f()
        a[at] = keep
        assert abs((up - down) / (2 * h) - g[at]) <= 1e-6 * max(1.0, abs(g[at])), at


def test_layer_norm_differences_and_library():
    rng = np.random.default_rng(0)
    x, w, b, dy = rng.normal(0.3, 1.5, (5, 7)), rng.normal(1, 0.2, 7), rng.normal(0, 1, 7), rng.normal(size=(5, 7))
    dx, dw, db = T.layer_norm_bwd(dy, x, w)
    f = lambda: float((T.layer_norm_fwd(x, w, b)[0] * dy).sum())
    _diff(f, x, dx, n=35)
    _diff(f, w, dw)
    _diff(f, b, db)
    want = torch.nn.functional.layer_norm(torch.from_numpy(x), (7,), torch.from_numpy(w), torch.from_numpy(b))
    assert np.allclose(T.layer_norm_fwd(x, w, b)[0], want.numpy(), rtol=0, atol=1e-12)
    # a row of one value and a constant row: the norm is the bias, no gradient reaches x
    y, _, _ = T.layer_norm_fwd(np.full((2, 1), 3.0), np.full(1, 2.0), np.full(1, 0.5))
    assert np.allclose(y, 0.5) and np.allclose(T.layer_norm_bwd(np.ones((2, 1)), np.full((2, 1), 3.0))[0], 0)


@pytest.mark.parametrize("kind", ACTS)
def test_linear_differences_and_library(kind):
    rng = np.random.default_rng(1)
    x, w, b, r, dy = (rng.normal(size=s) for s in ((4, 5), (5, 6), (6,), (4, 6), (4, 6)))
    y, z = T.linear_fwd(x, w, b, kind, r)
    dx, dw, db = T.linear_bwd(dy, x, w, z, kind)
    f = lambda: float((T.linear_fwd(x, w, b, kind, r)[0] * dy).sum())
    for a, g in ((x, dx), (w, dw), (b, db), (r, dy)):
        _diff(f, a, g)
    F = torch.nn.functional
    lib = {"none": lambda t: t, "relu": F.relu, "gelu": F.gelu, "gelu_tanh": lambda t: F.gelu(t, approximate="tanh"),
           "silu": F.silu}[kind]
    assert np.allclose(lib(torch.from_numpy(z)).numpy() + r, y, rtol=0, atol=1e-12)


def test_ce_differences_library_and_closed_forms():
    rng = np.random.default_rng(2)
    x, w = rng.normal(size=(6, 4)), rng.normal(size=(4, 9))
    labels = np.array([3, -100, 0, 8, 8, -100])
    got = T.ce(x, w, labels, dloss=0.7)
    f = lambda: 0.7 * T.ce(x, w, labels)["total"][0] / 4
    _diff(f, x, got["dx"], n=24)
    _diff(f, w, got["dw"], n=36)
    want = torch.nn.functional.cross_entropy(torch.from_numpy(x @ w), torch.from_numpy(labels), reduction="none")
    assert np.allclose(got["loss"], want.numpy(), rtol=0, atol=1e-12) and list(got["total"])[1] == 4
    # equal logits: ln V; nothing counted: no loss, no gradient
    assert np.allclose(T.ce(np.zeros((2, 4)), w, [1, 2])["loss"], math.log(9))
    none = T.ce(x, w, np.full(6, -100))
    assert none["total"][0] == 0 and not none["dx"].any() and not none["dw"].any()
    # per-row gradients
    g = rng.normal(size=6)
    rows = T.ce(x, w, labels, dloss=g)
    _diff(lambda: float((T.ce(x, w, labels)["loss"] * g).sum()), x, rows["dx"], n=24)


def test_kd_differences_library_and_closed_forms():
    rng = np.random.default_rng(3)
    x, w = rng.normal(size=(6, 4)), rng.normal(size=(4, 9))
    index = np.array([[3, 1, 0], [8, -1, -1], [-1, -1, -1], [2, 2, 5], [7, 0, 4], [1, 6, 2]])  # absent ones, one twice
    logits = rng.normal(size=(6, 3))
    logits[4, 1] = -np.inf
    got = T.kd(x, w, index, logits, 2.0, dloss=0.7)
    assert got["total"][1] == 5 and got["loss"][2] == 0 and not got["dx"][2].any()
    f = lambda: 0.7 * T.kd(x, w, index, logits, 2.0)["total"][0] / 5
    _diff(f, x, got["dx"], n=24)
    _diff(f, w, got["dw"], n=36)
    # one entry is cross entropy with that label (at T = 1); all V entries are the divergence of the two softmaxes
    one = T.kd(x, w, index[:, :1], logits[:, :1])
    lab = T.ce(x, w, index[:, 0], ignore=-1)
    for k in ("loss", "dx", "dw"):
        assert np.allclose(one[k], lab[k], rtol=0, atol=1e-12)
    t = rng.normal(size=(6, 9))
    full = T.kd(x, w, np.tile(np.arange(9), (6, 1)), t, 3.0)
    want = 9 * torch.nn.functional.kl_div(torch.log_softmax(torch.from_numpy(x @ w / 3), 1),
                                          torch.softmax(torch.from_numpy(t / 3), 1), reduction="none").sum(1)
    assert np.allclose(full["loss"], want.numpy(), rtol=0, atol=1e-12)
    # the student's own logits teach nothing
    same = T.kd(x, w, np.tile(np.arange(9), (6, 1)), x @ w, 3.0)
    assert np.allclose(same["loss"], 0, atol=1e-12) and np.allclose(same["dx"], 0, atol=1e-12)
