"""Layer norm, forward and backward, against the float64 oracle (GPU).

Bounds, element by element.  A sum over a row of N values runs over at most 32 terms in
a lane, 6 steps across lanes and 16 wavefronts: each value is off by at most 54 half
steps of fp32, below 2^-18 of the sum of magnitudes.  The mean is off by that times
mean|x|, so xh = (x - mean) rstd by 2^-18 rstd mean|x| and, from the variance, the products and
the square root, by 2^-17 |xh|.  The sums down the columns run over at most M / groups
rows in a lane, 16 slots, then groups / 32 and 32 terms."""
import numpy as np
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import DTYPES, check, note, padded, rounded
from oracle import train as oracle

pytestmark = pytest.mark.gpu


def _xh_bound(x, rstd, xh):
    return 2.0 ** -18 * rstd[:, None] * np.abs(x).mean(1, keepdims=True) + 2.0 ** -17 * np.abs(xh)


def _run(M, N, dt, weight=True, bias=True, eps=1e-5, strided=False, shift=0.3, seed=0):
    rng = np.random.default_rng(seed + M + N)
    x, xr = rounded(rng, (M, N), dt, 1.5, shift)
    dy, dyr = rounded(rng, (M, N), dt)
    w, wr = rounded(rng, (N,), dt, 0.2, 1.0) if weight else (None, None)
    b, br = rounded(rng, (N,), dt, 0.2) if bias else (None, None)
    note(f"layer norm M={M} N={N} {dt} weight={weight} bias={bias} strided={strided}")
    out = dx = None
    bufs = []
    if strided:
        x, dy = padded(x)[0], padded(dy, 3)[0]
        for _ in range(2):
            v, buf = padded(torch.zeros(M, N, dtype=dt, device="cuda"), 7, 9.0)
            bufs.append(buf)
            out, dx = (v, dx) if out is None else (out, v)
    y, mean, rstd = fbl.layer_norm_fwd(x, w, b, eps, out=out)
    dx, dw, db = fbl.layer_norm_bwd(dy, x, mean, rstd, w, dx=dx)
    torch.cuda.synchronize()
    yr, mr, rr = oracle.layer_norm_fwd(xr, wr, br, eps)
    dxr, dwr, dbr = oracle.layer_norm_bwd(dyr, xr, wr, eps)
    xh = (xr - mr[:, None]) * rr[:, None]
    one = np.ones(N) if wr is None else np.abs(wr)
    near = _xh_bound(xr, rr, xh)
    check("mean", mean, mr, 2.0 ** -18 * np.abs(xr).mean(1))
    check("rstd", rstd, rr, rr * (2.0 ** -17 + 2.0 ** -17 * rr * np.abs(xr).mean(1)))
    check("y", y, yr, near * one + 2.0 ** -22 * (np.abs(xh * one) + (0 if br is None else np.abs(br))))
    g = np.abs(dyr) * one
    terms = g + g.mean(1, keepdims=True) + np.abs(xh) * (g * np.abs(xh)).mean(1, keepdims=True)
    check("dx", dx, dxr, rr[:, None] * (2.0 ** -16 * terms + near * (g * np.abs(xh)).mean(1, keepdims=True)
                                        + np.abs(xh) * (g * near).mean(1, keepdims=True)))
    depth = (min(M, 64 + M / 512) + 64) * 2.0 ** -24
    check("dw", dw, dwr, depth * np.abs(dyr * xh).sum(0) + (np.abs(dyr) * near).sum(0))
    check("db", db, dbr, depth * np.abs(dyr).sum(0))
    for buf in bufs:  # nothing written between the rows or behind the last
        assert torch.all(buf[:, N:] == 9.0) and torch.all(buf[-1] == 9.0)
    return x, dy, w, b, y, mean, rstd, dx, dw, db


WIDTHS = [1, 2, 7, 32, 128, 129, 256, 511, 512, 768, 1001, 1024, 1025, 2048, 2049, 4096, 4100, 8192, 8195, 16384]


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("N", WIDTHS)
def test_widths(N, dt):
    _run(37, N, DTYPES[dt])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("M,N", [(1, 768), (2, 16384), (3, 64), (8191, 128), (2050, 1000), (700, 4096), (1025, 5001)])
def test_rows(M, N, dt):
    _run(M, N, DTYPES[dt])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("weight,bias", [(False, False), (True, False), (False, True)])
def test_without_weight_or_bias(weight, bias, dt):
    _run(19, 300, DTYPES[dt], weight, bias)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("N", [5, 128, 130, 1000, 2047, 5000])
def test_strided_rows(N, dt):
    """Rows with gaps between them (of odd width: rows of any element alignment)."""
    _run(23, N, DTYPES[dt], strided=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_far_mean(dt):
    """A mean of 1000 deviations: the variance is taken about it."""
    _run(9, 1024, DTYPES[dt], shift=1500.0)


def test_constant_rows_and_non_finite_ones():
    x = torch.zeros(4, 96, device="cuda")
    x[0] = 2.5
    x[1] = torch.arange(96)
    x[2, 5] = float("inf")
    x[3, 7] = float("nan")
    w, b = torch.full((96,), 2.0, device="cuda"), torch.full((96,), 0.5, device="cuda")
    y, mean, rstd = fbl.layer_norm_fwd(x, w, b)
    dx, _, _ = fbl.layer_norm_bwd(torch.ones_like(x), x, mean, rstd, w)
    torch.cuda.synchronize()
    assert torch.equal(y[0], b) and mean[0] == 2.5
    assert torch.isfinite(y[1]).all() and torch.isfinite(dx[:2]).all()
    assert torch.isnan(y[2:]).all()  # each row keeps its own


def test_repeatable_and_partial_gradients():
    rng = np.random.default_rng(4)
    x, _ = rounded(rng, (3000, 777), torch.bfloat16)
    dy, _ = rounded(rng, (3000, 777), torch.bfloat16)
    w, _ = rounded(rng, (777,), torch.bfloat16)
    y, mean, rstd = fbl.layer_norm_fwd(x, w)
    a = fbl.layer_norm_bwd(dy, x, mean, rstd, w)
    b = fbl.layer_norm_bwd(dy, x, mean, rstd, w)
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    c = fbl.layer_norm_bwd(dy, x, mean, rstd, w, need_weight=False)
    d = fbl.layer_norm_bwd(dy, x, mean, rstd, w, need_weight=False, need_bias=False)
    assert c[1] is None and torch.equal(c[2], a[2]) and torch.equal(c[0], a[0])
    assert d[1] is None and d[2] is None and torch.equal(d[0], a[0])


def test_autograd_matches_the_calls():
    from paper_2607_21624_amd import autograd as ag
    rng = np.random.default_rng(5)
    x, w, b, dy = (rounded(rng, s, torch.bfloat16)[0] for s in ((4, 50, 320), (320,), (320,), (4, 50, 320)))
    leaves = [t.clone().requires_grad_(True) for t in (x, w, b)]
    y = ag.layer_norm(*leaves)
    y.backward(dy)
    y2, mean, rstd = fbl.layer_norm_fwd(x.view(-1, 320), w, b)
    want = fbl.layer_norm_bwd(dy.view(-1, 320), x.view(-1, 320), mean, rstd, w)
    assert torch.equal(y, y2.view_as(y))
    for t, g in zip(leaves, want):
        assert torch.equal(t.grad, g.view_as(t))
    with pytest.raises(fbl.FblError):
        ag.layer_norm(leaves[0]).sum().backward()  # a broadcast gradient is refused, as everywhere


def test_streams_and_graph():
    """On another stream without a workspace of the caller's, and replayed in a graph."""
    rng = np.random.default_rng(6)
    x, _ = rounded(rng, (512, 1000), torch.bfloat16)
    dy, _ = rounded(rng, (512, 1000), torch.bfloat16)
    w, _ = rounded(rng, (1000,), torch.bfloat16)
    step = lambda s=None: (lambda f: f[:1] + fbl.layer_norm_bwd(dy, x, f[1], f[2], w, stream=s))(
        fbl.layer_norm_fwd(x, w, w, stream=s))
    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    raw = step(side.cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(want, got, raw))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for _ in range(3):
        for t in out:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out))
        assert torch.isfinite(torch.randn(1 << 16, device="cuda").sum())
