"""Softmax cross entropy and distillation on a linear head, forward and backward,
against the float64 oracle (GPU).

Bounds, element by element.  A logit's sum of K terms in fp32 is off by at most
(K + 16) 2^-24 of the sum of magnitudes, zb.  lse is off by the largest zb / T of its
row, by the sums of exponentials (at most 64 terms in a lane, then some tens: 2^-17 of the
sum) and by its own rounding.  q = exp(z / T - lse) is off by the sum of those,
relative; dz = g T (q - p) besides by half a step of the storage type, which dx and
dw carry through their sums of magnitudes."""
import numpy as np
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import DTYPES, HALF, check, note, padded, rounded
from oracle import train as oracle

pytestmark = pytest.mark.gpu


def _inputs(M, K, V, dt, table, seed=0, scale=2.0):
    rng = np.random.default_rng(seed + 13 * M + 5 * K + V)
    x, xr = rounded(rng, (M, K), dt)
    if table:
        w, wr = rounded(rng, (V, K), dt, scale * K ** -0.5)
        return rng, x, xr, w.t(), wr.T
    w, wr = rounded(rng, (K, V), dt, scale * K ** -0.5)
    return rng, x, xr, w, wr


def _check(got, ref, xr, wr, T, dt, target, g):
    """got: dict of tensors (loss, lse, total, dx, dw); target [M, V]: the targets' weights; g [M]: the factors."""
    K = xr.shape[1]
    zb = (K + 16) * 2.0 ** -24 * (np.abs(xr) @ np.abs(wr))
    lb = zb.max(1) / T + 2.0 ** -17 + 2.0 ** -21 * np.abs(ref["lse"])
    check("lse", got["lse"], ref["lse"], lb)
    on = target.sum(1) > 0
    z = xr @ wr / T
    terms = np.abs(np.where(target > 0, np.log(np.where(target > 0, target, 1.0)), 0) * target).sum(1) + (target * np.abs(z)).sum(1)
    loss_b = T * T * np.where(on, lb + (target * zb).sum(1) / T + 2.0 ** -18 * (terms + np.abs(ref["lse"]) + 1), 0)
    check("loss", got["loss"], ref["loss"], loss_b)
    check("total", got["total"], ref["total"], np.array([loss_b.sum() + len(on) * 2.0 ** -24 * np.abs(ref["loss"]).sum(), 0]))
    q = np.exp(z - ref["lse"][:, None])
    gT = np.abs(g * T)[:, None] * on[:, None]
    dz = gT * np.abs(q - target)
    off = gT * (q * (zb / T + lb[:, None] + 2.0 ** -20) + 2.0 ** -21 * target)
    each = off + (HALF[dt] * (dz + off) if dt == torch.bfloat16 else 0) + 2.0 ** -22 * dz
    V, M = wr.shape[1], len(xr)
    if got.get("dx") is not None:
        check("dx", got["dx"], ref["dx"], (V + 16) * 2.0 ** -24 * ((dz + each) @ np.abs(wr.T)) + each @ np.abs(wr.T))
    if got.get("dw") is not None:
        check("dw", got["dw"], ref["dw"], (M + 16) * 2.0 ** -24 * (np.abs(xr.T) @ (dz + each)) + np.abs(xr.T) @ each)


def _ce(M, K, V, dt, table, ignored=0.2, dloss=0.7, seed=0, x=None):
    rng, x, xr, w, wr = _inputs(M, K, V, dt, table, seed)
    labels = rng.integers(0, V, M)
    labels[rng.random(M) < ignored] = -100
    note(f"ce M={M} K={K} V={V} {dt} table={table}")
    lab = torch.from_numpy(labels).cuda()
    rows = np.ndim(dloss) > 0
    g = torch.tensor(dloss, dtype=torch.float32, device="cuda")
    mean = torch.full((), float("nan"), device="cuda")
    loss, lse, total = fbl.linear_ce_fwd(x, w, lab, mean=mean)
    dx, dw = fbl.linear_ce_bwd(g, x, w, lab, lse, None if rows else total)
    torch.cuda.synchronize()
    assert dw.stride() == w.stride()
    ref = oracle.ce(xr, wr, labels, dloss=dloss)
    target = np.zeros((M, V))
    on = labels >= 0
    target[np.nonzero(on)[0], labels[on]] = 1
    factor = np.asarray(dloss) if rows else np.full(M, dloss / max(on.sum(), 1))
    got = dict(loss=loss, lse=lse, total=total, dx=dx, dw=dw)
    _check(got, ref, xr, wr, 1.0, dt, target, factor)
    assert abs(float(mean) - float(total[0]) / max(int(on.sum()), 1)) <= 2.0 ** -23 * abs(float(mean))
    return x, w, lab, got


def _kd(M, K, V, top, dt, table, T, absent=0.3, dloss=0.7, seed=0, ldt=None):
    rng, x, xr, w, wr = _inputs(M, K, V, dt, table, seed)
    index = np.stack([rng.choice(V, top, replace=V < top) for _ in range(M)])
    index[rng.random((M, top)) < absent] = -1
    index[rng.random(M) < absent / 2] = -1  # rows without a teacher
    logits, lr = rounded(rng, (M, top), ldt or dt, 2.0, 5.0)
    note(f"kd M={M} K={K} V={V} top={top} {dt} table={table} T={T}")
    idx = torch.from_numpy(index).cuda()
    loss, lse, prob, total = fbl.linear_kd_fwd(x, w, idx, logits, T)
    dx, dw = fbl.linear_kd_bwd(torch.tensor(dloss, device="cuda"), x, w, idx, prob, lse, T, total)
    torch.cuda.synchronize()
    ref = oracle.kd(xr, wr, index, lr, T, dloss=dloss)
    check("prob", prob, ref["prob"], 2.0 ** -19 * ref["prob"])
    target = np.zeros((M, V))
    for j in range(top):
        np.add.at(target, (np.arange(M), np.maximum(index[:, j], 0)), ref["prob"][:, j])
    got = dict(loss=loss, lse=lse, total=total, dx=dx, dw=dw)
    _check(got, ref, xr, wr, T, dt, target, np.full(M, dloss / max(ref["total"][1], 1)))
    return x, w, idx, logits, prob, got


SHAPES = [(1, 64, 64), (1, 512, 5000), (7, 72, 1000), (32, 128, 1024), (33, 64, 2056), (64, 200, 1000), (65, 64, 776),
          (128, 64, 3000), (129, 264, 520), (300, 96, 4104), (515, 64, 264)]


@pytest.mark.parametrize("table", [False, True])
@pytest.mark.parametrize("M,K,V", SHAPES)
def test_ce_bf16(M, K, V, table):
    _ce(M, K, V, torch.bfloat16, table)


@pytest.mark.parametrize("M,K,V", [(5, 64, 1), (40, 64, 3), (100, 72, 1001), (300, 96, 2113), (1, 128, 50257)])
def test_ce_bf16_table_of_any_length(M, K, V):
    _ce(M, K, V, torch.bfloat16, True, ignored=0.0 if M < 10 else 0.2)


@pytest.mark.parametrize("table", [False, True])
@pytest.mark.parametrize("M,K,V", [(1, 1, 1), (1, 33, 700), (3, 17, 2), (64, 65, 1003), (65, 64, 333), (200, 130, 259)])
def test_ce_f32(M, K, V, table):
    _ce(M, K, V, torch.float32, table, ignored=0.0 if M < 10 else 0.2)


@pytest.mark.parametrize("table", [False, True])
@pytest.mark.parametrize("M,K,V,dt", [(4, 3600, 288, "bf16"), (16, 8192, 128, "bf16"), (100, 2048, 1000, "bf16"),
                                      (300, 4096, 1000, "bf16"), (2, 64, 60824, "bf16"), (5, 1100, 300, "f32"),
                                      (70, 1030, 333, "f32"), (130, 40, 5003, "f32"), (3, 40, 30011, "f32")])
def test_ce_few_tiles(M, K, V, dt, table):
    """A contraction split among a tile's wavefronts, a vocabulary among workgroups: many planes of dX."""
    _ce(M, K, V, DTYPES[dt], table)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_ce_per_row_gradient(dt):
    _ce(70, 64, 520, DTYPES[dt], True, dloss=np.random.default_rng(0).normal(size=70).astype(np.float32))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("table", [False, True])
@pytest.mark.parametrize("M,K,V,top,T", [(1, 64, 72, 1, 1.0), (33, 64, 1000, 8, 2.0), (100, 128, 520, 50, 4.0),
                                         (300, 72, 2056, 32, 1.0), (20, 64, 400, 200, 0.5)])
def test_kd(M, K, V, top, T, table, dt):
    _kd(M, K, V, top, DTYPES[dt], table, T, absent=0.0 if M == 1 else 0.3)


def test_kd_other_logits_type_and_many_entries():
    _kd(40, 64, 1032, 5, torch.bfloat16, True, 2.0, ldt=torch.float32)
    _kd(40, 64, 1032, 5, torch.float32, False, 2.0, ldt=torch.bfloat16)
    _kd(9, 64, 2048, 1024, torch.bfloat16, False, 3.0)


def test_kd_with_one_entry_is_cross_entropy():
    x, w, lab, ce = _ce(90, 64, 640, torch.bfloat16, True)
    idx = torch.where(lab == -100, -1, lab)[:, None]
    logits = torch.randn(90, 1, device="cuda")
    loss, lse, prob, total = fbl.linear_kd_fwd(x, w, idx, logits)
    dx, dw = fbl.linear_kd_bwd(torch.tensor(0.7, device="cuda"), x, w, idx, prob, lse, total=total)
    for a, b in ((loss, ce["loss"]), (lse, ce["lse"]), (total, ce["total"]), (dx, ce["dx"]), (dw, ce["dw"])):
        assert torch.equal(a, b)


def test_kd_repeated_entries_add_up():
    """The same entry twice counts with both weights."""
    x, w = torch.randn(3, 16, device="cuda"), torch.randn(16, 40, device="cuda")
    idx = torch.tensor([[7, 7, 3], [5, -1, 5], [0, 0, 0]], device="cuda")
    logits = torch.randn(3, 3, device="cuda")
    loss, lse, prob, total = fbl.linear_kd_fwd(x, w, idx, logits, 2.0)
    dx, dw = fbl.linear_kd_bwd(torch.ones((), device="cuda"), x, w, idx, prob, lse, 2.0, total)
    ref = oracle.kd(x.cpu().numpy(), w.cpu().numpy(), idx.cpu().numpy(), logits.cpu().numpy(), 2.0, dloss=1.0)
    for a, k in ((loss, "loss"), (dx, "dx"), (dw, "dw")):  # sums of at most 40 fp32 terms of size 10
        check(k, a, ref[k], 1e-4)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("table", [False, True])
def test_nothing_counts(table, dt):
    """Every label ignored, no teacher anywhere, teacher logits of -inf: no loss, a mean of 0, gradients of 0."""
    _, x, _, w, _ = _inputs(40, 64, 200, DTYPES[dt], table)
    lab = torch.full((40,), -100, device="cuda")
    mean = torch.ones((), device="cuda")
    loss, lse, total = fbl.linear_ce_fwd(x, w, lab, mean=mean)
    dx, dw = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, total)
    assert not loss.any() and not total.any() and mean == 0 and not dx.any() and not dw.any() and torch.isfinite(lse).all()
    idx = torch.full((40, 4), -1, device="cuda")
    idx[::2] = 3
    logits = torch.full((40, 4), float("-inf"), device="cuda")
    logits[1::2] = 1.0
    loss, lse, prob, total = fbl.linear_kd_fwd(x, w, idx, logits, 2.0, mean=mean)
    dx, dw = fbl.linear_kd_bwd(torch.ones((), device="cuda"), x, w, idx, prob, lse, 2.0, total)
    assert not loss.any() and not prob.any() and not total.any() and mean == 0 and not dx.any() and not dw.any()


def test_ignored_rows_may_hold_anything():
    """x of ignored rows inf and nan: no other row's loss or gradient sees them but dW, whose sum over rows does not
    (their dz is 0) unless x itself is not finite."""
    _, x, _, w, _ = _inputs(40, 64, 200, torch.bfloat16, True)
    lab = torch.arange(40, device="cuda")
    lab[5] = lab[20] = -100
    clean = fbl.linear_ce_fwd(x, w, lab)
    want = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, clean[1], clean[2])
    x[5], x[20] = 3e38, -3e38  # logits overflow to inf and nan
    loss, lse, total = fbl.linear_ce_fwd(x, w, lab)
    dx, dw = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, total)
    assert torch.equal(loss, clean[0]) and torch.equal(total, clean[2])
    assert torch.equal(dx, want[0]) and torch.equal(dw, want[1])


@pytest.mark.parametrize("bad", [200, 1 << 40, -1])
def test_labels_outside_the_vocabulary_show(bad):
    _, x, _, w, _ = _inputs(40, 64, 200, torch.bfloat16, True)
    lab = torch.arange(40, device="cuda")
    lab[7] = bad
    loss, lse, total = fbl.linear_ce_fwd(x, w, lab)
    dx, _ = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, total)
    assert torch.isnan(loss[7]) and torch.isnan(total[0]) and total[1] == 40 and torch.isnan(dx[7]).all()
    keep = torch.arange(40, device="cuda") != 7
    assert torch.isfinite(loss[keep]).all() and torch.isfinite(dx[keep]).all() and torch.isfinite(lse).all()
    if bad < 0:
        return
    idx = torch.stack([lab, (lab + 1) % 200], 1)
    loss, lse, prob, total = fbl.linear_kd_fwd(x, w, idx, torch.ones(40, 2, device="cuda"))
    dx, _ = fbl.linear_kd_bwd(torch.ones((), device="cuda"), x, w, idx, prob, lse, total=total)
    assert torch.isnan(loss[7]) and torch.isnan(dx[7]).all() and torch.isfinite(loss[keep]).all() and torch.isfinite(dx[keep]).all()


@pytest.mark.parametrize("scale", [60.0, 3000.0])
def test_far_logits(scale):
    """Logits of hundreds and of ten thousands: the exponentials are relative to the row's maximum."""
    rng, x, xr, w, wr = _inputs(50, 64, 328, torch.float32, False, scale=scale)
    labels = rng.integers(0, 328, 50)
    lab = torch.from_numpy(labels).cuda()
    loss, lse, total = fbl.linear_ce_fwd(x, w, lab)
    ref = oracle.ce(xr, wr, labels)
    zb = (64 + 16) * 2.0 ** -24 * (np.abs(xr) @ np.abs(wr)).max(1)
    check("lse", lse, ref["lse"], zb + 2.0 ** -17 + 2.0 ** -21 * np.abs(ref["lse"]))
    check("loss", loss, ref["loss"], 2 * zb + 2.0 ** -17 + 2.0 ** -21 * np.abs(ref["lse"]) + 2.0 ** -22 * np.abs(xr @ wr).max(1))


@pytest.mark.parametrize("dt,gap", [("bf16", 8), ("f32", 3)])
@pytest.mark.parametrize("table", [False, True])
def test_strided_operands(table, dt, gap):
    """Views with gaps of NaN between their rows give the contiguous call's bits; nothing is written into the gaps."""
    dt = DTYPES[dt]
    _, x, _, w, _ = _inputs(90, 72, 520, dt, table)
    rows = w.t() if table else w  # the stored rows
    lab = torch.arange(90, device="cuda") * 5
    one = torch.ones((), device="cuda")
    a = fbl.linear_ce_fwd(x, w, lab)
    want = fbl.linear_ce_bwd(one, x, w, lab, a[1], a[2])
    xs, (ws, _) = padded(x, gap)[0], padded(rows, gap)
    (dxs, dxb), (dws, dwb) = padded(torch.zeros_like(x), gap, 5.0), padded(torch.zeros_like(rows), gap, 5.0)
    view = lambda t: t.t() if table else t
    b = fbl.linear_ce_fwd(xs, view(ws), lab)
    fbl.linear_ce_bwd(one, xs, view(ws), lab, b[1], b[2], dx=dxs, dw=view(dws))
    torch.cuda.synchronize()
    assert all(torch.equal(s, t) for s, t in zip(a, b))
    assert torch.equal(dxs, want[0]) and torch.equal(view(dws), want[1])
    for buf, t in ((dxb, x), (dwb, rows)):
        assert torch.all(buf[:, t.shape[1]:] == 5.0) and torch.all(buf[-1] == 5.0)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("table", [False, True])
def test_pieces_of_the_vocabulary(table, dt):
    """A dz of more than 128 MiB is made and used in pieces; against float64 on the card."""
    dt = DTYPES[dt]
    M, K, V = (2100, 64, 70000) if dt == torch.bfloat16 else (1100, 40, 70003)
    if not table:
        V = V // 8 * 8
    rng, x, _, w, _ = _inputs(M, K, V, dt, table)
    lab = torch.from_numpy(rng.integers(0, V, M)).cuda()
    lab[::9] = -100
    note(f"pieces {M} {K} {V} {dt} table={table}")
    loss, lse, total = fbl.linear_ce_fwd(x, w, lab)
    dx, dw = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, total)
    xd, wd = x.double(), w.double()
    z = xd @ wd
    lse_r = torch.logsumexp(z, 1)
    on = lab >= 0
    n = on.sum()
    z.sub_(lse_r[:, None]).exp_()
    z[torch.arange(M, device="cuda")[on], lab[on]] -= 1
    z *= (on / n)[:, None]
    dxr, dwr = z @ wd.t(), xd.t() @ z
    assert (lse - lse_r).abs().max() <= 2.0 ** -16
    half = HALF[dt]
    # dz's rounding through sums of magnitudes, the result's own; fp32 sums of V and M terms
    zabs = z.abs()
    for got, ref, mag, terms in ((dx, dxr, zabs @ wd.abs().t(), V), (dw, dwr, xd.abs().t() @ zabs, M)):
        bound = half * ref.abs() + mag * ((half if dt == torch.bfloat16 else 0) + 2.0 ** -15 + (terms + 16) * 2.0 ** -24)
        assert bool(((got.double() - ref).abs() <= bound).all())
    again = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, total)
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    one = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, total, need_dw=False)
    two = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, total, need_dx=False)
    assert torch.equal(one[0], dx) and one[1] is None and torch.equal(two[1], dw) and two[0] is None


def test_more_tiles_than_a_launch_holds():
    """2^20 rows of 2^19 logits: 2^23 tiles of 512 threads would be 2^32, one more than a launch may have.  64 rows'
    loss and dx against float64."""
    dt = torch.bfloat16
    M, K, V = 1 << 20, 8, 1 << 19
    note(f"ce M={M} K={K} V={V}")
    g = torch.Generator("cuda").manual_seed(5)
    x, w = (torch.randn(s, generator=g, device="cuda").to(dt) for s in ((M, K), (K, V)))
    lab = torch.randint(0, V, (M,), generator=g, device="cuda")
    loss, lse, total = fbl.linear_ce_fwd(x, w, lab)
    dx, _ = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, None, need_dw=False)
    at = torch.linspace(0, M - 1, 64, device="cuda").long()
    xd, wd, ld = x[at].double(), w.double(), lab[at]
    z = xd @ wd
    ref = torch.logsumexp(z, 1)
    picked = z.gather(1, ld[:, None])[:, 0]
    # K + 16 roundings of a logit, the sums of exponentials (2^-17), lse's and the loss' own
    zb = (K + 16) * 2.0 ** -24 * (xd.abs() @ wd.abs()).amax(1)
    bound = 2 * zb + 2.0 ** -17 + 2.0 ** -20 * (ref.abs() + picked.abs())
    assert bool(((loss[at].double() - (ref - picked)).abs() <= bound).all())
    z.sub_(ref[:, None]).exp_()
    z.scatter_add_(1, ld[:, None], torch.full((64, 1), -1.0, dtype=torch.float64, device="cuda"))
    want, mag = z @ wd.t(), z.abs() @ wd.abs().t()
    bound = HALF[dt] * want.abs() + mag * (HALF[dt] + 2.0 ** -15 + zb.amax() * 2 + (V + 16) * 2.0 ** -24)
    assert bool(((dx[at].double() - want).abs() <= bound).all())
    assert total[1] == M


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
def test_autograd(reduction):
    from paper_2607_21624_amd import autograd as ag
    B, S, K, V = 3, 21, 64, 200
    rng, x, xr, w, wr = _inputs(B * S, K, V, torch.bfloat16, True)
    labels = rng.integers(0, V, B * S)
    labels[::7] = -100
    lab = torch.from_numpy(labels).cuda()
    X, E = x.view(B, S, K).clone().requires_grad_(True), w.t().clone().requires_grad_(True)  # E: the table
    loss = ag.linear_cross_entropy(X, E.t(), lab.view(B, S), reduction=reduction)
    raw, lse, total = fbl.linear_ce_fwd(x, w, lab)
    if reduction == "none":
        assert loss.shape == (B, S)
        loss.sum().backward()  # a broadcast gradient: one number for all rows
    else:
        loss.backward()
    assert torch.equal(loss.reshape(-1), {"none": raw, "sum": total[:1], "mean": (total[0] / total[1])[None]}[reduction])
    dx, dw = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, w, lab, lse, total if reduction == "mean" else None)
    assert torch.equal(X.grad.view(-1, K), dx) and torch.equal(E.grad, dw.t())
    idx = torch.from_numpy(np.stack([rng.choice(V, 6, replace=False) for _ in range(B * S)])).cuda()
    logits = torch.randn(B, S, 6, device="cuda")
    X.grad = E.grad = None
    loss = ag.linear_distillation(X, E.t(), idx.view(B, S, 6), logits, 2.0, reduction)
    (loss.sum() if reduction == "none" else loss).backward()
    raw, lse, prob, total = fbl.linear_kd_fwd(x, w, idx, logits.view(-1, 6), 2.0)
    dx, dw = fbl.linear_kd_bwd(torch.ones((), device="cuda"), x, w, idx, prob, lse, 2.0, total if reduction == "mean" else None)
    assert torch.equal(X.grad.view(-1, K), dx) and torch.equal(E.grad, dw.t())
    # frozen head, frozen trunk
    for freeze in (X, E):
        a, b = (X.detach(), E.detach().requires_grad_(True)) if freeze is X else (X.detach().requires_grad_(True), E.detach())
        ag.linear_distillation(a, b.t(), idx.view(B, S, 6), logits, 2.0, reduction).sum().backward()
        assert torch.equal(a.grad.view(-1, K), dx) if freeze is E else torch.equal(b.grad, dw.t())


def test_differences():
    """The gradients against central differences of the library's own loss (fp32): the loss is smooth, a step of
    1/32 gives a difference good to h^2 / 6 of a third derivative (below 1) and to the loss' rounding over h."""
    rng, x, _, w, _ = _inputs(12, 16, 50, torch.float32, False)
    idx = torch.from_numpy(np.stack([rng.choice(50, 4, replace=False) for _ in range(12)])).cuda()
    logits = torch.randn(12, 4, device="cuda")
    loss, lse, prob, total = fbl.linear_kd_fwd(x, w, idx, logits, 2.0)
    dx, dw = fbl.linear_kd_bwd(torch.ones((), device="cuda"), x, w, idx, prob, lse, 2.0)
    h = 1.0 / 32
    for t, g in ((x, dx), (w, dw)):
        for i in rng.choice(t.numel(), 20, replace=False):
            at = np.unravel_index(i, tuple(t.shape))
            keep = t[at].item()
            side = []
            for s in (h, -h):
                t[at] = keep + s
                side.append(fbl.linear_kd_fwd(x, w, idx, logits, 2.0)[0].double().sum().item())
            t[at] = keep
            # per row 3 terms of 2^-20 of about 10 over 2 h; the third derivative sums over 12 rows of |x|^3 <= 40 / T
            assert abs((side[0] - side[1]) / (2 * h) - g[at].item()) <= 12 * 30 * 2.0 ** -20 / h + h * h / 6 * 12 * 20, at


def test_streams_and_graph():
    """Another stream without a workspace of the caller's; replays of a graph; two graphs with one workspace between
    them, replayed in turn."""
    rng, x, _, w, _ = _inputs(200, 128, 1000, torch.bfloat16, True)
    lab = torch.from_numpy(rng.integers(0, 1000, 200)).cuda()
    idx = torch.from_numpy(rng.integers(0, 1000, (200, 5))).cuda()
    logits = torch.randn(200, 5, device="cuda")
    one = torch.ones((), device="cuda")

    def ce(stream=None, ws=None):
        f = fbl.linear_ce_fwd(x, w, lab, stream=stream, workspace=ws)
        return f + fbl.linear_ce_bwd(one, x, w, lab, f[1], f[2], stream=stream, workspace=ws)

    def kd(stream=None, ws=None):
        f = fbl.linear_kd_fwd(x, w, idx, logits, 2.0, stream=stream, workspace=ws)
        return f + fbl.linear_kd_bwd(one, x, w, idx, f[2], f[1], 2.0, f[3], stream=stream, workspace=ws)
    want = [ce(), kd()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = [ce(side), kd(side)]
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(s, t) for s, t in zip(a, b))
    shared = torch.empty(fbl.linear_loss_workspace(x, w, 5), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for f in (ce, kd):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(f(ws=shared))
        graphs.append(g)
    for _ in range(3):
        for g, out, ref in zip(graphs, outs, want):
            for t in out:
                t.fill_(float("nan"))
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(s, t) for s, t in zip(out, ref))
            assert torch.isfinite(torch.randn(1 << 16, device="cuda").sum())
