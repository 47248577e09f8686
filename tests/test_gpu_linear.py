"""Linear layers with bias, activation and residual, forward and backward, and the
feed-forward part built from two, against the float64 oracle (GPU).

Bounds, element by element.  A product's sum of K terms in fp32 is off by at most (K + 16)
2^-24 of the sum of magnitudes (bf16 products are exact in fp32).  Half a rounding step
for y and, where the backward reads it, for z: z's reaches dz = dy act'(z) through
|act''| <= 2, and dz's own rounding reaches dx and dw through their sums of magnitudes.  The bf16
activations are good to 2^-20 of their argument (reciprocal and exp2 to an ulp each,
the distribution function to 1.5e-7)."""
import numpy as np
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import DTYPES, HALF, check, note, padded, rounded
from oracle import train as oracle

pytestmark = pytest.mark.gpu
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _sum_bound(a, b):
    """Of the product a b in fp32."""
    return (a.shape[1] + 16) * 2.0 ** -24 * (np.abs(a) @ np.abs(b))


def _case(M, K, N, dt, act, bias, residual, seed=0):
    rng = np.random.default_rng(seed + M * 7 + K * 3 + N)
    x, xr = rounded(rng, (M, K), dt)
    w, wr = rounded(rng, (K, N), dt, K ** -0.5)
    b, br = rounded(rng, (N,), dt, 0.5) if bias else (None, None)
    r, rr = rounded(rng, (M, N), dt) if residual else (None, None)
    dy, dyr = rounded(rng, (M, N), dt)
    note(f"linear {M}x{K}x{N} {dt} {act} bias={bias} residual={residual}")
    return (x, w, b, r, dy), (xr, wr, br, rr, dyr)


def _check_fwd(y, z, ref, act, dt):
    xr, wr, br, rr, _ = ref
    yr, zr = oracle.linear_fwd(xr, wr, br, act, rr)
    zb = _sum_bound(xr, wr) + 2.0 ** -23 * (np.abs(zr) + (0 if br is None else np.abs(br)))
    yb = 1.2 * zb + 2.0 ** -20 * np.abs(zr) + (0 if rr is None else 2.0 ** -22 * (np.abs(rr) + np.abs(zr)))
    if z is not None:
        check("z", z, zr, zb)
    check("y", y, yr, yb)
    return zr, zb


def _check_bwd(dx, dw, db, ref, zr, zb, act, dt, x_grad=None):
    xr, wr, _, _, dyr = ref
    dxr, dwr, dbr = oracle.linear_bwd(dyr, xr, wr, zr, act)
    half = HALF[dt]
    # what dz may be off by: z's rounding and bound, the derivative's own error, its rounding
    dz = np.abs(dyr * oracle.act_grad(zr, act))
    off = np.zeros_like(dz) if act == "none" else np.abs(dyr) * (2.0 * (half * np.abs(zr) + zb) + 2.0 ** -20 * (1 + np.abs(zr)))
    if act == "relu":  # a step: z within its bound of 0 may fall on either side, and nothing else matters
        off = np.where(np.abs(zr) <= zb, np.abs(dyr), 0.0)
    rounding = 0 if act == "none" else half
    each = off + rounding * (dz + off)
    if dx is not None:
        check("dx", dx, dxr, _sum_bound(dz + each, wr.T) + each @ np.abs(wr.T))
    if dw is not None:
        check("dw", dw, dwr, _sum_bound(xr.T, dz + each) + np.abs(xr.T) @ each)
    if db is not None:
        M = len(dyr)
        check("db", db, dbr, (M + 16) * 2.0 ** -24 * dz.sum(0) + off.sum(0))


def _run(M, K, N, dt, act, bias=True, residual=True, tile=-1):
    (x, w, b, r, dy), ref = _case(M, K, N, dt, act, bias, residual)
    z = torch.full((M, N), float("nan"), dtype=dt, device="cuda") if act != "none" else None
    y = fbl.linear_fwd(x, w, b, act, r, z=z, tile=tile)
    dx, dw, db = fbl.linear_bwd(dy, x, w, z, act)
    torch.cuda.synchronize()
    zr, zb = _check_fwd(y, z, ref, act, dt)
    _check_bwd(dx, dw, db, ref, zr, zb, act, dt)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", [(1, 64, 64), (3, 256, 520), (33, 72, 200), (200, 512, 264), (1001, 128, 96), (257, 1024, 768), (9000, 72, 136)])
def test_bf16(M, K, N, act):
    _run(M, K, N, torch.bfloat16, act)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 300, 77), (5, 63, 130), (130, 257, 65), (333, 100, 1), (64, 512, 768)])
def test_f32(M, K, N, act):
    _run(M, K, N, torch.float32, act)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
def test_parts(bias, residual, dt):
    _run(70, 96, 136, DTYPES[dt], "gelu", bias, residual)
    _run(70, 96, 136, DTYPES[dt], "none", bias, residual)


@pytest.mark.parametrize("M", [1, 2, 3, 4, 5, 7, 8, 9, 16, 17, 32, 33])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_few_tokens(M, dt):
    dt = DTYPES[dt]
    for K, N, act in ((4096, 1032, "silu"), (264, 4104, "none"), (64, 8, "gelu"), (2048, 64, "gelu_tanh")):
        (x, w, b, r, _), ref = _case(M, K, N, dt, act, True, True)
        _check_fwd(fbl.linear_fwd(x, w, b, act, r), None, ref, act, dt)
        z = torch.empty((M, N), dtype=dt, device="cuda")
        _check_fwd(fbl.linear_fwd(x, w, None, act, None, z=z), z, (ref[0], ref[1], None, None, None), act, dt)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_few_tokens_shared_contraction(dt):
    """A contraction that several workgroups share: strided operands, a share that ends inside a step, and the same
    bits with the caller's workspace, an allocated one and on another stream."""
    dt = DTYPES[dt]
    for M, K, N in ((1, 4104, 260), (13, 5000, 132), (32, 8200, 64)):
        if dt == torch.float32:
            K, N = K + 1, N + 1
        (x, w, b, r, _), ref = _case(M, K, N, dt, "gelu", True, True)
        x, w, r = (padded(t, 4 if N % 8 == 4 and dt == torch.bfloat16 and t is not x else 8)[0] for t in (x, w, r))
        need = fbl.linear_fwd_workspace(x, w)
        assert need > 0 and need % (M * N * 4) == 0
        z, zbuf = padded(torch.zeros(M, N, dtype=dt, device="cuda"), 4 if N % 8 == 4 else 8, 7.0)
        new = lambda: padded(torch.zeros(M, N, dtype=dt, device="cuda"), 4 if N % 8 == 4 else 8, 7.0)[0]
        y = fbl.linear_fwd(x, w, b, "gelu", r, z=z, out=new())
        _check_fwd(y, z, ref, "gelu", dt)
        assert torch.all(zbuf[:, N:] == 7.0) and torch.all(zbuf[-1] == 7.0)
        ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")  # nan, if it were read before it is written
        assert torch.equal(y, fbl.linear_fwd(x, w, b, "gelu", r, out=new(), workspace=ws[:need]))
        assert torch.all(ws[need:] == 0xff)
        side, got = torch.cuda.Stream(), new()
        side.wait_stream(torch.cuda.current_stream())
        fbl.linear_fwd(x, w, b, "gelu", r, out=got, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(y, got)
        with pytest.raises(fbl.FblError):
            fbl.linear_fwd(x, w, b, "gelu", r, out=new(), workspace=ws[:need - 16])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_few_tokens_shared_data_gradient(act, dt):
    """dx of a few tokens over a long contraction, plain and times act'(x_z), into views with gaps."""
    dt = DTYPES[dt]
    for M, K, N in ((1, 260, 4104), (20, 132, 5000), (64, 64, 8200)):
        if dt == torch.float32:
            K, N = K + 1, N + 1
        rng = np.random.default_rng(M)
        xz, xzr = rounded(rng, (M, K), dt)
        w, wr = rounded(rng, (K, N), dt, N ** -0.5)
        dy, dyr = rounded(rng, (M, N), dt)
        note(f"shared dx {M}x{K}x{N} {dt} {act}")
        gap = 4 if K % 8 == 4 else 8
        dx, buf = padded(torch.zeros(M, K, dtype=dt, device="cuda"), gap, 7.0)
        x = padded(xz, gap)[0]
        got, _, _ = fbl.linear_bwd(dy, x, w, dx=dx, need_dw=False, need_bias=False, x_act=act, x_z=x if act != "none" else None)
        d = oracle.act_grad(xzr, act)
        prod = dyr @ wr.T
        check("dx", got, prod * d, np.abs(d) * _sum_bound(dyr, wr.T) + np.abs(prod) * 2.0 ** -20 * (1 + np.abs(xzr)))
        assert torch.all(buf[:, K:] == 7.0) and torch.all(buf[-1] == 7.0)
        # with the bias' gradient too, and without a workspace of the caller's or with one
        ws = torch.full((fbl.linear_bwd_workspace(xz, w),), 0xff, dtype=torch.uint8, device="cuda")
        a = fbl.linear_bwd(dy, x, w, dx=padded(torch.zeros(M, K, dtype=dt, device="cuda"), gap)[0], need_dw=False, x_act=act,
                           x_z=x if act != "none" else None, workspace=ws)
        assert torch.equal(a[0], got)
        check("db", a[2], dyr.sum(0), (M + 16) * 2.0 ** -24 * np.abs(dyr).sum(0))


@pytest.mark.parametrize("tile", range(21))
def test_every_tile(tile):
    """Ragged against every tile: a partial last step, partial rows and columns, into NaN."""
    M, K, N = 301, 360, 268
    (x, w, b, r, _), ref = _case(M, K, N, torch.bfloat16, "gelu", True, True)
    w, r = padded(w, 4)[0], padded(r, 4)[0]  # rows of 268 are 16-byte aligned 272 apart
    z, zbuf = padded(torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"), 4, 7.0)
    out, obuf = padded(torch.zeros(M, N, dtype=torch.bfloat16, device="cuda"), 4, 7.0)
    fbl.linear_fwd(x, w, b, "gelu", r, out=out, z=z, tile=tile)
    _check_fwd(out, z, ref, "gelu", torch.bfloat16)
    for buf in (zbuf, obuf):
        assert torch.all(buf[:, N:] == 7.0) and torch.all(buf[-1] == 7.0)


@pytest.mark.parametrize("dt,gap", [("bf16", 8), ("f32", 3)])
@pytest.mark.parametrize("act", ["none", "gelu_tanh"])
def test_strided_operands(dt, gap, act):
    """Every matrix a view with gaps of NaN between its rows; bit for bit the contiguous call."""
    dt = DTYPES[dt]
    (x, w, b, r, dy), _ = _case(75, 88, 104, dt, act, True, True)
    z = torch.empty_like(dy) if act != "none" else None
    y = fbl.linear_fwd(x, w, b, act, r, z=z)
    want = fbl.linear_bwd(dy, x, w, z, act)
    view = lambda t: None if t is None else padded(t, gap)[0]
    z2 = view(z)
    y2 = fbl.linear_fwd(view(x), view(w), b, act, view(r), z=z2, out=view(torch.zeros_like(y)))
    got = fbl.linear_bwd(view(dy), view(x), view(w), z2, act, dx=view(torch.zeros_like(x)), dw=view(torch.zeros_like(w)))
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and (z is None or torch.equal(z, z2))
    assert all(torch.equal(a, c) for a, c in zip(want, got))


def test_wanted_gradients_alone_are_the_same():
    (x, w, b, r, dy), _ = _case(100, 64, 72, torch.bfloat16, "silu", True, False)
    z = torch.empty_like(dy)
    fbl.linear_fwd(x, w, b, "silu", z=z)
    full = fbl.linear_bwd(dy, x, w, z, "silu")
    for keep in range(3):
        flags = dict(need_dx=keep == 0, need_dw=keep == 1, need_bias=keep == 2)
        got = fbl.linear_bwd(dy, x, w, z, "silu", **flags)
        for i in range(3):
            assert (torch.equal(got[i], full[i]) if i == keep else got[i] is None)
    assert fbl.linear_bwd(dy, x, w, None, need_dx=False, need_dw=False, need_bias=False) == (None, None, None)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,N", [(300, 96, 384), (77, 264, 64)])
def test_gradient_of_the_previous_pre_activation(M, K, N, act, dt):
    """dx as the gradient of x_z, x = x_act(x_z): the product times act'(x_z)."""
    dt = DTYPES[dt]
    rng = np.random.default_rng(M + N)
    xz, xzr = rounded(rng, (M, K), dt)
    (x, w, _, _, dy), ref = _case(M, K, N, dt, "none", False, False)
    got = fbl.linear_bwd(dy, x, w, need_dw=False, need_bias=False, x_act=act, x_z=xz)[0]
    d = oracle.act_grad(xzr, act)
    prod = ref[4] @ ref[1].T
    check("dxz", got, prod * d, np.abs(d) * _sum_bound(ref[4], ref[1].T) + np.abs(prod) * 2.0 ** -20 * (1 + np.abs(xzr)))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("M,K,N", [(8200, 64, 72), (9001, 132, 260), (4099, 256, 264), (20000, 8, 16)])
def test_small_weights_of_many_tokens(M, K, N, dt):
    """dw with its contraction shared among workgroups; written between the guards of a larger matrix."""
    dt = DTYPES[dt]
    (x, w, _, _, dy), ref = _case(M, K, N, dt, "none", False, False)
    row = lambda t: padded(t, 8 + -t.shape[1] % 8)[0]
    view, buf = padded(torch.zeros(K, N, dtype=dt, device="cuda"), 8 + -N % 8, 9.0)
    dx, dw, _ = fbl.linear_bwd(row(dy), row(x), row(w), dw=view, need_dx=False, need_bias=False)
    check("dw", dw, ref[0].T @ ref[4], _sum_bound(ref[0].T, ref[4]))
    assert bool((buf[:, N:] == 9.0).all()) and bool((buf[-1] == 9.0).all())
    again = fbl.linear_bwd(row(dy), row(x), row(w), dw=row(torch.zeros_like(w)), need_dx=False, need_bias=False)[1]
    assert torch.equal(again, dw)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("act", ["none", "gelu"])
@pytest.mark.parametrize("M,K,N", [(1, 264, 64), (3, 12, 264), (40, 1028, 8200), (77, 260, 64), (300, 100, 384), (1000, 2052, 200),
                                   (4096, 512, 264), (2000, 8192, 64), (1001, 8192, 64), (2050, 1000, 2048),
                                   (2050, 256, 512), (1000, 64, 256), (4100, 8200, 128), (4096, 4096, 1024)])
def test_sums_of_the_data_gradient(M, K, N, act, dt):
    """dxbias: dx summed over its rows before its rounding, with tiles of every kind and with shared contractions.
    Each dx is off by its product's bound and act's; then M fp32 additions."""
    dt = DTYPES[dt]
    rng = np.random.default_rng(M + N)
    xz, xzr = rounded(rng, (M, K), dt)
    (x, w, _, _, dy), ref = _case(M, K, N, dt, "none", False, False)
    buf = torch.full((K + 8,), 7.0, dtype=dt, device="cuda")
    new = lambda t: padded(t, -K % 8)[0]  # rows of whole 16-byte chunks
    kw = dict(need_dw=False, need_bias=False, x_act=act, x_z=None if act == "none" else new(xz))
    dx = fbl.linear_bwd(dy, new(x), w, dx=new(torch.zeros_like(x)), dxbias=buf[:K], **kw)[0]
    assert torch.equal(dx, fbl.linear_bwd(dy, new(x), w, dx=new(torch.zeros_like(x)), **kw)[0]) or (dt == torch.float32 and act == "none")
    assert bool((buf[K:] == 7.0).all())
    d = oracle.act_grad(xzr, act) if act != "none" else np.ones_like(xzr)
    prod = ref[4] @ ref[1].T
    off = np.abs(d) * _sum_bound(ref[4], ref[1].T) + (0 if act == "none" else np.abs(prod) * 2.0 ** -20 * (1 + np.abs(xzr)))
    dxr = prod * d
    check("dx", dx, dxr, off)
    check("dxbias", buf[:K], dxr.sum(0), off.sum(0) + (M + 16) * 2.0 ** -24 * np.abs(dxr).sum(0))
    again = torch.empty(K, dtype=dt, device="cuda")
    fbl.linear_bwd(dy, new(x), w, dx=new(torch.zeros_like(x)), dxbias=again, **kw)
    assert torch.equal(again, buf[:K])
    # an infinite weight: that column alone, infinite of one sign, and no nan from rows behind the last
    w[1, 0] = float("inf")
    fbl.linear_bwd(dy.abs() + 1, new(x), w, dx=new(torch.zeros_like(x)), need_dw=False, need_bias=False, dxbias=again)
    assert again[1] == float("inf") and bool(again.isfinite().sum() == K - 1)


@pytest.mark.parametrize("act", ACTS)
def test_extreme_pre_activations(act):
    """z far out on both sides: saturated values and derivatives of 0 and 1, nothing non-finite."""
    for dt in (torch.bfloat16, torch.float32):
        z = torch.tensor([[-3e4, -300.0, -50.0, -12.0, 0.0, 12.0, 300.0, 3e4]], device="cuda").to(dt)
        eye = torch.eye(8, device="cuda").to(dt)
        y = fbl.linear_fwd(z, eye, None, act)
        g = fbl.linear_bwd(torch.ones_like(z), torch.zeros_like(z), eye, need_dw=False, need_bias=False, x_act=act, x_z=z)[0]
        zr = z.double().cpu().numpy()
        with np.errstate(over="ignore"):
            check("act", y, oracle.act(zr, act), 2.0 ** -20 * np.minimum(np.abs(zr), 1.0))
            check("act'", g, oracle.act_grad(zr, act), 2.0 ** -20)


def test_autograd_and_mlp():
    from paper_2607_21624_amd import autograd as ag
    B, S, K, N = 3, 41, 64, 256
    M = B * S
    rng = np.random.default_rng(9)
    dt = torch.bfloat16
    t = {n: rounded(rng, s, dt, sc)[0] for n, s, sc in (("x", (B, S, K), 1), ("w1", (K, N), K ** -0.5), ("b1", (N,), 0.3),
                                                      ("w2", (N, K), N ** -0.5), ("b2", (K,), 0.3), ("r", (B, S, K), 1),
                                                      ("dy", (B, S, K), 1))}
    leaf = {k: v.clone().requires_grad_(True) for k, v in t.items()}
    # linear through autograd equals the calls
    y = ag.linear(leaf["x"], leaf["w1"], leaf["b1"], "gelu")
    y.backward(torch.ones_like(y))
    z = torch.empty(M, N, dtype=dt, device="cuda")
    y2 = fbl.linear_fwd(t["x"].view(M, K), t["w1"], t["b1"], "gelu", z=z)
    want = fbl.linear_bwd(torch.ones_like(y2), t["x"].view(M, K), t["w1"], z, "gelu")
    assert torch.equal(y.view(M, N), y2)
    for k, g in zip(("x", "w1", "b1"), want):
        assert torch.equal(leaf[k].grad, g.view_as(t[k]))
        leaf[k].grad = None
    # mlp: forward the two layers; its gradients the oracle's, dz1 rounded once
    y = ag.mlp(leaf["x"], leaf["w1"], leaf["b1"], leaf["w2"], leaf["b2"], "gelu", leaf["r"])
    y.backward(t["dy"])
    h = fbl.linear_fwd(t["x"].view(M, K), t["w1"], t["b1"], "gelu", z=z)
    y2 = fbl.linear_fwd(h, t["w2"], t["b2"], residual=t["r"].view(M, K))
    assert torch.equal(y.view(M, K), y2)
    db1 = torch.empty(N, dtype=dt, device="cuda")
    dz, dw2, db2 = fbl.linear_bwd(t["dy"].view(M, K), h, t["w2"], x_act="gelu", x_z=z, dxbias=db1)
    dx, dw1, _ = fbl.linear_bwd(dz, t["x"].view(M, K), t["w1"])
    for k, g in (("x", dx), ("w1", dw1), ("b1", db1), ("w2", dw2), ("b2", db2), ("r", t["dy"])):
        assert torch.equal(leaf[k].grad, g.view_as(t[k])), k
    f = {k: v.double().cpu().numpy().reshape(-1, v.shape[-1]) if v.dim() > 1 else v.double().cpu().numpy() for k, v in t.items()}
    hr, zr = oracle.linear_fwd(f["x"], f["w1"], f["b1"], "gelu")
    dzr = (f["dy"] @ f["w2"].T) * oracle.act_grad(zr, "gelu")
    for k, ref in (("x", dzr @ f["w1"].T), ("w1", f["x"].T @ dzr), ("b1", dzr.sum(0)), ("w2", hr.T @ f["dy"])):
        got = leaf[k].grad.double().cpu().numpy().reshape(ref.shape)
        # two roundings of half a step in the chain, each seen through a sum of terms of random sign
        assert np.abs(got - ref).max() <= 4 * HALF[dt] * np.abs(ref).max(), k
    # frozen parts
    frozen = {k: v.detach() for k, v in leaf.items()}
    for k in ("x", "b1", "w2", "r"):
        one = {**frozen, k: t[k].clone().requires_grad_(True)}
        ag.mlp(one["x"], one["w1"], one["b1"], one["w2"], one["b2"], "gelu", one["r"]).backward(t["dy"])
        assert torch.equal(one[k].grad, leaf[k].grad), k


def test_residual_alone_needs_no_product():
    from paper_2607_21624_amd import autograd as ag
    (x, w, b, r, dy), _ = _case(40, 64, 64, torch.bfloat16, "relu", True, True)
    r.requires_grad_(True)
    ag.linear(x, w, b, "relu", r).backward(dy)
    assert torch.equal(r.grad, dy)


def test_stream_graph_and_repeats():
    (x, w, b, r, dy), _ = _case(515, 264, 392, torch.bfloat16, "gelu", True, True)
    z = torch.empty_like(dy)

    def step(stream=None):
        y = fbl.linear_fwd(x, w, b, "gelu", r, z=z, stream=stream)
        return (y,) + fbl.linear_bwd(dy, x, w, z, "gelu", stream=stream)
    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(want, got))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step()
    for _ in range(3):
        for t in out:
            t.fill_(float("nan"))
        z.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(want, out))
        assert torch.isfinite(torch.randn(1 << 16, device="cuda").sum())


def test_another_stream_shares_no_memory_with_queued_work():
    """Results and workspaces of a call on another stream do not come out of blocks that the current stream's queue
    still writes: temporaries of a long queue are freed, then a call goes to a stream that does not wait for it."""
    (x, w, b, r, dy), _ = _case(16, 4096, 512, torch.bfloat16, "gelu", True, True)
    want = fbl.linear_fwd(x, w, b, "gelu", r)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for stream in (side, side.cuda_stream):
        a = torch.randn(2048, 2048, device="cuda")
        for _ in range(20):  # some milliseconds
            a = a @ a * 1e-3
        for size in (want.numel() * 2, fbl.linear_fwd_workspace(x, w)):
            torch.full((size,), 0xff, dtype=torch.uint8, device="cuda")  # queued behind, freed at once
        got = fbl.linear_fwd(x, w, b, "gelu", r, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(got, want)
