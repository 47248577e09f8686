"""Gated layers, forward and backward, and the feed-forward part built from them, against the float64 oracle (GPU).

Bounds, element by element, as in test_gpu_linear.py: a product's sum of K terms in fp32 is off by at most (K + 16)
2^-24 of the sum of magnitudes, activations by 2^-20 of their argument, their derivatives by 2^-20 (1 + |argument|), and |act'|
<= 1.2, |act''| <= 1 (relu's is a step: a gate within its bound of 0 may fall on either side).  h = act(gate) up and the factors
are made from unrounded sums and rounded once each: factors of bf16 layers are off by 2^-11 of themselves where they are
within 2^13 of the largest of their eight, and by 2^-24 of that otherwise.  The backward reads factors that are given, so that
the oracle has the same."""
import numpy as np
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import DTYPES, check, note, padded, rounded
from oracle import gated_block as oracle
from oracle.train import act as act_of, act_grad

pytestmark = pytest.mark.gpu
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _sum_bound(a, b):
    return (a.shape[1] + 16) * 2.0 ** -24 * (np.abs(a) @ np.abs(b))


def _inputs(M, K, F, N, dt, bias, seed=0):
    rng = np.random.default_rng(seed + M * 7 + K * 3 + F)
    note(f"gated {M}x{K}x{F} -> {N} {dt} bias={bias}")
    x, w, wd, f, dy = (rounded(rng, s, dt, k) for s, k in (((M, K), 1.0), ((K, 2 * F), K ** -0.5), ((F, N), N ** -0.5),
                                                           ((M, 2 * F), 1.5), ((M, N), 1.0)))
    if dt == torch.bfloat16:
        kept = oracle.keep_factors(f[1])
        f = torch.from_numpy(kept.view(np.int16)).cuda().view(torch.bfloat16), oracle.kept_factors(kept)
    b = rounded(rng, (2 * F,), dt, 0.5) if bias else (None, None)
    return x, w, b, wd, f, dy


def _check_fwd(h, f, x, w, b, act):
    hr, zr = oracle.gated_fwd(x, w, b, act)
    F = hr.shape[1]
    zb = _sum_bound(x, w) + 2.0 ** -23 * (np.abs(zr) + (0 if b is None else np.abs(b)))
    gate, up = zr[:, :F], zr[:, F:]
    gb = 1.2 * zb[:, :F] + 2.0 ** -20 * np.abs(gate)  # of act(gate)
    if f is not None:
        slope = np.abs(act_grad(gate, act))
        sb = zb[:, :F] + 2.0 ** -20 * (1 + np.abs(gate))
        if act == "relu":
            sb = np.where(np.abs(gate) <= zb[:, :F], 1.0, 0.0)
        fr = oracle.gated_factors(zr, act)
        fb = np.concatenate([zb[:, F:] * (slope + sb) + np.abs(up) * sb, gb], axis=1) + 2.0 ** -23 * np.abs(fr)
        if f.dtype == torch.bfloat16:
            got = torch.from_numpy(oracle.kept_factors(f.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)))
            top = np.repeat((np.abs(fr) + fb).reshape(len(fr), -1, 8).max(-1), 8, axis=-1)
            off = np.abs(got.numpy() - fr) - fb - np.maximum(2.0 ** -11 * (np.abs(fr) + fb), 2.0 ** -24 * top)
            assert np.all(off <= 0), ("factors", np.unravel_index(np.argmax(off), off.shape), off.max())
        else:
            check("factors", f, fr, fb)
    check("h", h, hr, gb * np.abs(up) + (np.abs(act_of(gate, act)) + gb) * zb[:, F:] + 2.0 ** -23 * np.abs(hr))


def _check_bwd(dz, db, dy, wd, f):
    dh = dy @ wd.T
    ref = oracle.gated_bwd(dh, f)
    dhb = _sum_bound(dy, wd.T)
    bound = np.concatenate([dhb, dhb], axis=1) * np.abs(f) + 2.0 ** -23 * np.abs(ref)
    check("dz", dz, ref, bound)
    if db is not None:
        check("dbias", db, ref.sum(0), (len(dy) + 16) * 2.0 ** -24 * (np.abs(ref) + bound).sum(0) + bound.sum(0))


def _run(M, K, F, N, dt, act, bias=True, tile=-1):
    (x, xr), (w, wr), (b, br), (wd, wdr), (f, fr), (dy, dyr) = _inputs(M, K, F, N, dt, bias)
    fo = torch.full((M, 2 * F), float("nan"), dtype=dt, device="cuda")
    h = fbl.gated_fwd(x, w, b, act, factors=fo, tile=tile)
    only = fbl.gated_fwd(x, w, b, act, tile=tile)
    dz, db = fbl.gated_bwd(dy, wd, f, need_bias=bias, tile=tile)
    torch.cuda.synchronize()
    _check_fwd(h, fo, xr, wr, br, act)
    assert torch.equal(h, only)
    _check_bwd(dz, db, dyr, wdr, fr)
    assert (db is None) == (not bias)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,F,N", [(1, 64, 64, 64), (3, 256, 264, 72), (33, 72, 200, 136), (200, 512, 136, 256),
                                     (1001, 128, 48, 96), (257, 1024, 384, 768), (9000, 72, 8, 64)])
def test_bf16(M, K, F, N, act):
    _run(M, K, F, N, torch.bfloat16, act)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,K,F,N", [(1, 1, 1, 1), (1, 300, 39, 7), (5, 63, 65, 130), (130, 257, 33, 100), (333, 100, 1, 3),
                                     (64, 512, 384, 512), (700, 129, 257, 65)])
def test_f32(M, K, F, N, act):
    _run(M, K, F, N, torch.float32, act)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_without_bias(dt):
    _run(70, 96, 136, 104, DTYPES[dt], "silu", bias=False)


@pytest.mark.parametrize("tile", range(21))
def test_every_tile(tile):
    """Ragged against every tile: partial last steps, rows and columns; nothing written between the rows."""
    M, K, F, N = 301, 360, 280, 168
    (x, xr), (w, wr), (b, br), (wd, wdr), (f, fr), (dy, dyr) = _inputs(M, K, F, N, torch.bfloat16, True)
    x, w, wd, fin, dy = (padded(t, 8)[0] for t in (x, w, wd, f, dy))
    h, hbuf = padded(torch.zeros(M, F, dtype=torch.bfloat16, device="cuda"), 8, 7.0)
    fo, fbuf = padded(torch.zeros(M, 2 * F, dtype=torch.bfloat16, device="cuda"), 8, 7.0)
    dz, dbuf = padded(torch.zeros(M, 2 * F, dtype=torch.bfloat16, device="cuda"), 8, 7.0)
    fbl.gated_fwd(x, w, b, "gelu", out=h, factors=fo, tile=tile)
    _, db = fbl.gated_bwd(dy, wd, fin, dz=dz, tile=tile)
    torch.cuda.synchronize()
    _check_fwd(h, fo, xr, wr, br, "gelu")
    _check_bwd(dz, db, dyr, wdr, fr)
    for buf, n in ((hbuf, F), (fbuf, 2 * F), (dbuf, 2 * F)):
        assert torch.all(buf[:, n:] == 7.0) and torch.all(buf[-1] == 7.0)


@pytest.mark.parametrize("M", [1, 2, 3, 5, 8, 16, 17, 33, 64, 65, 100, 128])
@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_few_tokens(M, dt):
    dt = DTYPES[dt]
    for K, F, act in ((4096, 264, "silu"), (264, 1032, "none"), (64, 8, "gelu"), (2048, 64, "gelu_tanh")):
        _run(M, K, F, K, dt, act)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_shared_contractions(dt):
    """Contractions that several workgroups share, strided and ragged; the same bits with the caller's workspace, an allocated
    one and on another stream; nothing read from the workspace before it is written or written behind it."""
    dt = DTYPES[dt]
    for M, K, F, N in ((1, 4104, 136, 4104), (13, 5000, 64, 5000), (64, 8200, 72, 8200)):
        odd = dt == torch.float32
        (x, xr), (w, wr), (b, br), (wd, wdr), (f, fr), (dy, dyr) = _inputs(M, K + odd, F + odd, N + odd, dt, True)
        F = F + odd
        x, w, wd, f, dy = (padded(t, 8)[0] for t in (x, w, wd, f, dy))
        new = lambda n: padded(torch.zeros(M, n, dtype=dt, device="cuda"), 8, 7.0)
        need, back = fbl.gated_fwd_workspace(x, w), fbl.gated_bwd_workspace(dy, wd)
        assert need > 0 and need % (M * 2 * F * 4) == 0
        (h, hbuf), (fo, fbuf), (dz, dbuf) = new(F), new(2 * F), new(2 * F)
        fbl.gated_fwd(x, w, b, "silu", out=h, factors=fo)
        _, db = fbl.gated_bwd(dy, wd, f, dz=dz)
        _check_fwd(h, fo, xr, wr, br, "silu")
        _check_bwd(dz, db, dyr, wdr, fr)
        for buf, n in ((hbuf, F), (fbuf, 2 * F), (dbuf, 2 * F)):
            assert torch.all(buf[:, n:] == 7.0) and torch.all(buf[-1] == 7.0)
        ws = torch.full((max(need, back) + 64,), 0xff, dtype=torch.uint8, device="cuda")
        assert torch.equal(h, fbl.gated_fwd(x, w, b, "silu", out=new(F)[0], workspace=ws[:need]))
        assert torch.all(ws[need:] == 0xff)
        again = fbl.gated_bwd(dy, wd, f, dz=new(2 * F)[0], workspace=ws[:back])
        assert torch.equal(again[0], dz) and torch.equal(again[1], db) and torch.all(ws[max(need, back):] == 0xff)
        alone = fbl.gated_bwd(dy, wd, f, dz=new(2 * F)[0], need_bias=False)
        assert torch.equal(alone[0], dz) and alone[1] is None
        side, got = torch.cuda.Stream(), new(F)[0]
        side.wait_stream(torch.cuda.current_stream())
        fbl.gated_fwd(x, w, b, "silu", out=got, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(h, got)
        for call in (lambda: fbl.gated_fwd(x, w, b, "silu", workspace=ws[:need - 16]),
                     lambda: fbl.gated_bwd(dy, wd, f, workspace=ws[:back - 16])):
            with pytest.raises(fbl.FblError):
                call()


@pytest.mark.parametrize("tile", range(21))
def test_tiles_of_few_tokens(tile):
    """A named tile shares no contraction, also where AUTO does: it writes its own rows of partial sums, and nothing behind the
    workspace."""
    for M, F, N in ((1, 264, 4096), (2, 136, 4104), (3, 264, 4096), (33, 136, 2056), (128, 72, 8192)):
        _, _, _, (wd, wdr), (f, fr), (dy, dyr) = _inputs(M, 64, F, N, torch.bfloat16, False)
        need = fbl.gated_bwd_workspace(dy, wd)
        ws = torch.full((need + 65536,), 0xff, dtype=torch.uint8, device="cuda")
        dz, db = fbl.gated_bwd(dy, wd, f, tile=tile, workspace=ws[:need])
        torch.cuda.synchronize()
        assert torch.all(ws[need:] == 0xff)
        _check_bwd(dz, db, dyr, wdr, fr)
        again = fbl.gated_bwd(dy, wd, f, tile=tile)
        assert torch.equal(again[0], dz) and torch.equal(again[1], db)


@pytest.mark.parametrize("dt,gap", [("bf16", 8), ("f32", 3)])
def test_strided_operands(dt, gap):
    """Every matrix a view with gaps of NaN between its rows; bit for bit the contiguous call."""
    dt = DTYPES[dt]
    (x, _), (w, _), (b, _), (wd, _), (f, _), (dy, _) = _inputs(75, 88, 104, 72, dt, True)
    fo = torch.empty_like(f)
    h = fbl.gated_fwd(x, w, b, "gelu_tanh", factors=fo)
    dz, db = fbl.gated_bwd(dy, wd, f)
    view = lambda t: padded(t, gap)[0]
    fv = view(torch.zeros_like(fo))
    assert torch.equal(h, fbl.gated_fwd(view(x), view(w), b, "gelu_tanh", factors=fv, out=view(torch.zeros_like(h))))
    got = fbl.gated_bwd(view(dy), view(wd), view(f), dz=view(torch.zeros_like(dz)))
    assert torch.equal(fv, fo) and torch.equal(got[0], dz) and torch.equal(got[1], db)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_infinite_weights_stay_in_their_columns(dt):
    """An infinity in the last up column reaches that column of h alone, whatever the tiles read past the halves' ends."""
    dt = DTYPES[dt]
    (x, _), (w, _), (b, _), _, _, _ = _inputs(40, 64, 72, 64, dt, True)
    clean = fbl.gated_fwd(x, w, b)
    for col, hit in ((143, 71), (72, 0), (71, 71)):
        bad = w.clone()
        bad[:, col] = float("inf")
        got = fbl.gated_fwd(x, bad, b)
        keep = torch.arange(72, device="cuda") != hit
        assert torch.equal(got[:, keep], clean[:, keep]) and not torch.isfinite(got[:, hit]).any()


def test_factors_of_any_size():
    """Every exponent keeps its digits, an element far below its neighbours what their exponent leaves it, and a factor that is
    not finite leaves its eight so; a few tokens' as a tile's."""
    dt = torch.bfloat16
    eye = torch.eye(16, dtype=dt, device="cuda")
    for M in (16, 200):
        rows = torch.arange(M, device="cuda") % 16
        x = eye[rows].contiguous()
        for up in (1.0, 2.0 ** 100, 2.0 ** -120, 2.0 ** -131, 3e38):
            w = torch.zeros(16, 48, dtype=dt, device="cuda")
            w[:, :24] = torch.linspace(-3, 3, 16 * 24, device="cuda").view(16, 24).to(dt)
            w[:, 24:] = (torch.linspace(0.1, 1, 16 * 24, device="cuda").view(16, 24) * up).to(dt)
            w[3, 24 + 9] = 0
            f = torch.empty(M, 48, dtype=dt, device="cuda")
            h = fbl.gated_fwd(x, w, None, "none", factors=f)  # factors: up, gate, exactly within 8 digits
            got = oracle.kept_factors(f.view(torch.int16).cpu().numpy().view(np.uint16))
            want = torch.cat([w[:, 24:], w[:, :24]], 1)[rows].double().cpu().numpy()
            top = np.repeat(np.abs(want).reshape(M, -1, 8).max(-1), 8, axis=-1)
            assert np.all(np.abs(got - want) <= 2.0 ** -24 * top) and torch.isfinite(h.float()[3]).all()
    for bad in (float("inf"), float("-inf"), float("nan")):
        for M in (16, 200):
            w = torch.ones(16, 48, dtype=dt, device="cuda")
            w[5, 24 + 10] = bad  # of up, the gate's factor
            x = eye[torch.arange(M, device="cuda") % 16].contiguous()
            f = torch.empty(M, 48, dtype=dt, device="cuda")
            fbl.gated_fwd(x, w, None, "none", factors=f)
            dz, _ = fbl.gated_bwd(torch.ones(M, 16, dtype=dt, device="cuda"), torch.ones(24, 16, dtype=dt, device="cuda"), f)
            keep = torch.ones(M, 48, dtype=torch.bool, device="cuda")
            # (0 times an infinite weight: the other rows' products with that column are nan)
            keep[:, 8:16] = False
            assert torch.all(dz[keep] == 16) and not torch.isfinite(dz[:, 8:16]).any()


@pytest.mark.parametrize("M", [40, 300])
@pytest.mark.parametrize("size", [2.0 ** 10, 2.0 ** 16, 2.0 ** 22])
def test_gradients_beside_outlier_columns(size, M):
    """One up column of eight is `size` times its neighbours, and so is its gate's factor: dw of the gates against float64, column
    by column as the factors' format has it.  A neighbour's factor keeps 2^-11 of itself, or 2^-24 of the outlier's; dz is
    rounded once, and its products with x are summed in fp32."""
    dt = torch.bfloat16
    K, F, N = 72, 64, 80
    rng = np.random.default_rng(17)
    note(f"outlier columns of {size}, {M} tokens")
    x, xr = rounded(rng, (M, K), dt)
    w1 = rng.standard_normal((K, 2 * F)) * K ** -0.5
    w1[:, F + 3::8] *= size
    w1 = torch.from_numpy(w1.astype(np.float32)).to(dt)
    w, wr = w1.cuda(), w1.double().numpy()
    (wd, wdr), (dy, dyr) = rounded(rng, (F, N), dt, N ** -0.5), rounded(rng, (M, N), dt)
    f = torch.empty(M, 2 * F, dtype=dt, device="cuda")
    fbl.gated_fwd(x, w, None, "silu", factors=f)
    dz, _ = fbl.gated_bwd(dy, wd, f, need_bias=False)
    _, dw, _ = fbl.linear_bwd(dz, x, w, need_dx=False, need_bias=False)
    _, zr = oracle.gated_fwd(xr, wr, None, "silu")
    fr = oracle.gated_factors(zr, "silu")[:, :F]
    zb = _sum_bound(xr, wr) + 2.0 ** -23 * np.abs(zr)
    gate, up = zr[:, :F], zr[:, F:]
    sb = zb[:, :F] + 2.0 ** -20 * (1 + np.abs(gate))
    fb = zb[:, F:] * (np.abs(act_grad(gate, "silu")) + sb) + np.abs(up) * sb + 2.0 ** -23 * np.abs(fr)
    top = np.repeat((np.abs(fr) + fb).reshape(M, -1, 8).max(-1), 8, axis=-1)
    fb = fb + np.maximum(2.0 ** -11 * (np.abs(fr) + fb), 2.0 ** -24 * top)
    dh = dyr @ wdr.T
    zg = dh * fr
    zgb = _sum_bound(dyr, wdr.T) * (np.abs(fr) + fb) + np.abs(dh) * fb
    zgb = zgb + 2.0 ** -8 * (np.abs(zg) + zgb)
    check("dw of the gates", dw[:, :F], xr.T @ zg,
          np.abs(xr).T @ zgb + (M + 16) * 2.0 ** -24 * (np.abs(xr).T @ (np.abs(zg) + zgb)), halves=1 + 2.0 ** -8)


def test_operands_near_the_limit():
    """Factors and dz of just below 2 GiB: the last rows are those of a call of their own, to the roundings of two tilings."""
    M, K, F = 262143, 64, 2040
    dt = torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(3)
    r = lambda *s, k=1.0: (torch.randn(s, generator=gen, device="cuda") * k).to(dt)
    x, w, wd, dy = r(M, K), r(K, 2 * F, k=K ** -0.5), r(F, K, k=K ** -0.5), r(M, K)
    note("gated near 2 GiB")
    f = torch.empty(M, 2 * F, dtype=dt, device="cuda")
    h = fbl.gated_fwd(x, w, None, "silu", factors=f)
    dz, db = fbl.gated_bwd(dy, wd, f)
    for at in (slice(M - 300, M), slice(131000, 131300)):
        few = torch.empty(300, 2 * F, dtype=dt, device="cuda")
        hs = fbl.gated_fwd(x[at].contiguous(), w, None, "silu", factors=few)
        ds, _ = fbl.gated_bwd(dy[at].contiguous(), wd, few)
        for a, b in ((h[at], hs), (dz[at], ds)):  # a rounding each way and sums of 64 terms in another order
            a, b = a.double(), b.double()
            assert torch.all((a - b).abs() <= 2.0 ** -7 * b.abs() + 1e-4)
    sums = torch.zeros(2 * F, dtype=torch.float64, device="cuda")
    most = torch.zeros(2 * F, dtype=torch.float64, device="cuda")
    for part in dz.split(32768):
        sums += part.double().sum(0)
        most += part.double().abs().sum(0)
    # dz rounded (2^-8 of each, added as they come) against sums of it unrounded in fp32 that are rounded once
    assert torch.all((db.double() - sums).abs() <= 2.0 ** -8 * (most + sums.abs()))


def test_silu_far_out():
    """act(gate) up where the gate saturates: no nan from the exponentials."""
    x = torch.eye(8, dtype=torch.bfloat16, device="cuda")
    gate = torch.tensor([-1e4, -200.0, -88.0, -1.0, 1.0, 88.0, 200.0, 1e4], dtype=torch.bfloat16, device="cuda")
    w = torch.cat([torch.diag(gate), torch.ones(8, 8, dtype=torch.bfloat16, device="cuda")], 1).contiguous()
    for act in ACTS:
        h = fbl.gated_fwd(x, w, None, act)
        with np.errstate(over="ignore"):
            ref = oracle.gated_fwd(np.eye(8), w.double().cpu().numpy(), None, act)[0]
        check(act, h, ref, 2.0 ** -18 * 1e-2)


# ------------------------------------------------------------------------ autograd
@pytest.mark.parametrize("dt,lead", [("bf16", (3, 20)), ("f32", (70,)), ("bf16", (1, 1))])
def test_autograd(dt, lead):
    from paper_2607_21624_amd import autograd as ag
    dtype = DTYPES[dt]
    K, F = 128, 328
    rng = np.random.default_rng(3)
    x, xr = rounded(rng, (*lead, K), dtype)
    w1, w1r = rounded(rng, (K, 2 * F), dtype, K ** -0.5)
    b1, b1r = rounded(rng, (2 * F,), dtype, 0.3)
    w2, w2r = rounded(rng, (F, K), dtype, F ** -0.5)
    b2, b2r = rounded(rng, (K,), dtype, 0.3)
    r, rr = rounded(rng, (*lead, K), dtype)
    dy, dyr = rounded(rng, (*lead, K), dtype)
    note(f"gated_mlp autograd {dt} {lead}")
    leaves = [t.requires_grad_(True) for t in (x, w1, b1, w2, b2, r)]
    y = ag.gated_mlp(x, w1, b1, w2, b2, act="silu", residual=r)
    assert y.shape == (*lead, K)
    got = torch.autograd.grad(y, leaves, dy)
    with torch.no_grad():  # bit for bit the explicit calls
        x2, r2, dy2 = (t.detach().view(-1, K) for t in (x, r, dy))
        f = torch.empty(x2.shape[0], 2 * F, dtype=dtype, device="cuda")
        h = fbl.gated_fwd(x2, w1, b1, "silu", factors=f)
        y2 = fbl.linear_fwd(h, w2, b2, residual=r2)
        dz, db1 = fbl.gated_bwd(dy2, w2, f)
        dx, dw1, _ = fbl.linear_bwd(dz, x2, w1, need_bias=False)
        _, dw2, db2 = fbl.linear_bwd(dy2, h, w2, need_dx=False)
    for a, b in zip((y, *got), (y2, dx, dw1, db1, dw2, db2, dy)):
        assert torch.equal(a.reshape(b.shape), b)
    p = [torch.from_numpy(t).requires_grad_(True) for t in (xr, w1r, b1r, w2r, b2r, rr)]
    zt = p[0] @ p[1] + p[2]
    yt = (torch.nn.functional.silu(zt[..., :F]) * zt[..., F:]) @ p[3] + p[4] + p[5]
    ref = torch.autograd.grad(yt, p, torch.from_numpy(dyr))
    # the factors, dz and h are rounded once each where they are kept: three half steps, and the result's own, of the largest value
    tol = 4 * 2.0 ** -8 if dt == "bf16" else 1e-5
    for a, b in zip((y, *got), (yt, *ref)):
        assert float((a.detach().double().cpu() - b.detach()).abs().max()) <= tol * float(b.detach().abs().max())
    # what is not needed is not made, and the rest stays
    for k in range(6):
        for t in leaves:
            t.requires_grad_(False)
        leaves[k].requires_grad_(True)
        y = ag.gated_mlp(x, w1, b1, w2, b2, act="silu", residual=r)
        (g,) = torch.autograd.grad(y, leaves[k], dy)
        assert torch.equal(g, got[k])
    for t in leaves:
        t.requires_grad_(False)
    assert not ag.gated_mlp(x, w1, b1, w2, b2, residual=r).requires_grad
    z = ag.gated_mlp(x.requires_grad_(True), w1, None, w2, None)
    z *= 2
    (g,) = torch.autograd.grad(z, x, dy, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_graph_replays():
    rng = np.random.default_rng(4)
    dtype = torch.bfloat16
    x, _ = rounded(rng, (130, 96), dtype)
    w1, _ = rounded(rng, (96, 2 * 136), dtype, 0.1)
    b1, _ = rounded(rng, (2 * 136,), dtype, 0.1)
    w2, _ = rounded(rng, (136, 96), dtype, 0.1)
    dy, _ = rounded(rng, (130, 96), dtype)
    f, h, dz = (torch.empty(130, n, dtype=dtype, device="cuda") for n in (272, 136, 272))
    db = torch.empty(272, dtype=dtype, device="cuda")
    ws = torch.empty(fbl.gated_bwd_workspace(dy, w2), dtype=torch.uint8, device="cuda")
    note("gated graph")

    def step():
        fbl.gated_fwd(x, w1, b1, factors=f, out=h)
        fbl.gated_bwd(dy, w2, f, dz=dz, dbias=db, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        x.copy_(rounded(rng, (130, 96), dtype)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (h, f, dz, db)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (h, f, dz, db)))
