"""The largest sizes: tables and activations whose offsets pass 31 and 32 bits, against
float64 on the card, a part of the rows where all would take too long (GPU)."""
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import DTYPES, HALF, note

pytestmark = pytest.mark.gpu


def _near(name, got, ref, bound):
    off = ((got.double() - ref).abs() - HALF[got.dtype] * ref.abs() - bound).max().item()
    assert off <= 0, f"{name}: {off} more than allowed"


def _parts(n, step=8192):
    return [slice(i, min(i + step, n)) for i in range(0, n, step)]


@pytest.mark.parametrize("dt,V,gap", [("bf16", 140001, 0), ("bf16", 131585, 8), ("f32", 70001, 0)])
def test_table_beyond_2_gib(dt, V, gap):
    """Read and written by pieces of whole rows.  Bounds as for smaller vocabularies: a logit's K + 16 roundings,
    2^-17 of the sums of exponentials, dz's rounding through sums of magnitudes."""
    dt = DTYPES[dt]
    M, K = 40, 8192
    note(f"table {V} x {K} {dt}")
    g = torch.Generator("cuda").manual_seed(V)
    table = torch.randn((V, K + gap), generator=g, device="cuda", dtype=torch.float32).mul_(K ** -0.5).to(dt)[:, :K]
    assert table.stride(0) * V * table.element_size() > 1 << 31
    x = torch.randn((M, K), generator=g, device="cuda").to(dt)
    lab = torch.randint(0, V, (M,), generator=g, device="cuda")
    lab[0], lab[1], lab[2] = V - 1, -100, 0
    loss, lse, total = fbl.linear_ce_fwd(x, table.t(), lab)
    dw = torch.full_like(table, float("nan"))
    dx, _ = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, table.t(), lab, lse, total, dw=dw.t())
    xd, on = x.double(), lab >= 0
    z = torch.cat([xd @ table[p].double().t() for p in _parts(V)], 1)
    zb = (K + 16) * 2.0 ** -24 * max((xd.abs() @ table[p].double().abs().t()).max().item() for p in _parts(V))
    lse_r = torch.logsumexp(z, 1)
    picked = z.gather(1, lab.clamp(min=0)[:, None])[:, 0]
    _near("lse", lse, lse_r, zb + 2.0 ** -17 + 2.0 ** -21 * lse_r.abs())
    _near("loss", loss, (lse_r - picked) * on, 2 * zb + 2.0 ** -17 + 2.0 ** -20 * (lse_r.abs() + picked.abs()))
    z.sub_(lse_r[:, None]).exp_()
    z[torch.arange(M, device="cuda")[on], lab[on]] -= 1
    z *= (on / on.sum())[:, None]
    each = (HALF[dt] if dt == torch.bfloat16 else 0) + 2 * zb + 2.0 ** -15
    want, mag = torch.zeros(M, K, dtype=torch.float64, device="cuda"), torch.zeros(M, K, dtype=torch.float64, device="cuda")
    for p in _parts(V):
        w = table[p].double()
        want += z[:, p] @ w
        mag += z[:, p].abs() @ w.abs()
        zt = z[:, p].t().contiguous()
        _near("dw", dw[p], zt @ xd, (zt.abs() @ xd.abs()) * (each + (M + 16) * 2.0 ** -24))
    _near("dx", dx, want, mag * (each + (V + 16) * 2.0 ** -24))


def test_layer_norm_beyond_4_gib():
    """Bounds: the sums over a row are off by 2^-18 of their magnitudes, xh by 2^-17 of itself and of mean |x| rstd;
    each of the sums down the columns runs over at most M / 256 rows in a lane, then 256 partial sums."""
    M, N, dt = (1 << 18) + 3, 8200, torch.bfloat16
    note(f"layer norm {M} x {N}")
    g = torch.Generator("cuda").manual_seed(1)
    x, dy = (torch.randn((M, N), generator=g, device="cuda", dtype=dt) for _ in range(2))
    w, b = (torch.randn(N, generator=g, device="cuda").to(dt) for _ in range(2))
    y, mean, rstd = fbl.layer_norm_fwd(x, w, b)
    dx, dw, db = fbl.layer_norm_bwd(dy, x, mean, rstd, w)
    sums = torch.zeros(4, N, dtype=torch.float64, device="cuda")
    wd, bd = w.double(), b.double()
    for p in _parts(M):
        xd, d = x[p].double(), dy[p].double()
        mu = xd.mean(1, keepdim=True)
        r = (xd.var(1, unbiased=False, keepdim=True) + 1e-5).rsqrt()
        xh = (xd - mu) * r
        sums += torch.stack([(d * xh).sum(0), d.sum(0), (d * xh).abs().sum(0), d.abs().sum(0)])
        if p.start % (1 << 16) and p.stop < M - 8192:
            continue  # rows at both ends and some between
        near = 2.0 ** -18 * r * xd.abs().mean(1, keepdim=True) + 2.0 ** -17 * xh.abs()
        _near("y", y[p], xh * wd + bd, near * wd.abs() + 2.0 ** -22 * ((xh * wd).abs() + bd.abs()))
        gr = d * wd
        c1, c2 = gr.mean(1, keepdim=True), (gr * xh).mean(1, keepdim=True)
        ga = gr.abs()
        terms = ga + ga.mean(1, keepdim=True) + xh.abs() * (ga * xh.abs()).mean(1, keepdim=True)
        bound = r * (2.0 ** -16 * terms + near * (ga * xh.abs()).mean(1, keepdim=True) + xh.abs() * (ga * near).mean(1, keepdim=True))
        _near("dx", dx[p], r * (gr - c1 - xh * c2), bound)
    depth = (M / 256 + 320) * 2.0 ** -24
    _near("dw", dw, sums[0], (depth + 2.0 ** -16) * sums[2] + 2.0 ** -17 * sums[3])
    _near("db", db, sums[1], depth * sums[3])


def test_linear_of_nearly_2_gib():
    """y, z and dz of 2146 MB: half a rounding step of y, of z through |act''| <= 2, of dz; sums of K, N and M terms."""
    M, K, N, dt = 134000, 16, 8008, torch.bfloat16
    assert 0 < (1 << 31) - M * N * 2 < 1 << 21
    note(f"linear {M} x {K} x {N}")
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.randn((M, K), generator=g, device="cuda").to(dt)
    w = torch.randn((K, N), generator=g, device="cuda").mul_(K ** -0.5).to(dt)
    b = torch.randn(N, generator=g, device="cuda").to(dt)
    dy = torch.randn((M, N), generator=g, device="cuda", dtype=dt)
    z = torch.empty((M, N), device="cuda", dtype=dt)
    y = fbl.linear_fwd(x, w, b, "silu", z=z)
    dx, dw, db = fbl.linear_bwd(dy, x, w, z, "silu")
    wd, half = w.double(), HALF[dt]
    sums = torch.zeros(K, N, dtype=torch.float64, device="cuda"), torch.zeros(K, N, dtype=torch.float64, device="cuda")
    dbr, dbb = (torch.zeros(N, dtype=torch.float64, device="cuda") for _ in range(2))
    for p in _parts(M):
        xd, d = x[p].double(), dy[p].double()
        zr = xd @ wd + b.double()
        zb = (K + 17) * 2.0 ** -24 * (xd.abs() @ wd.abs() + b.double().abs())
        s = torch.sigmoid(zr)
        _near("z", z[p], zr, zb)
        _near("y", y[p], zr * s, 1.2 * zb + 2.0 ** -20 * zr.abs())
        dz = d * s * (1 + zr * (1 - s))
        off = d.abs() * (2 * (half * zr.abs() + zb) + 2.0 ** -20 * (1 + zr.abs()))
        each = off + half * (dz.abs() + off)
        xt = xd.t().contiguous()
        sums[0].add_(xt @ dz)
        sums[1].add_(xt.abs() @ (each + (M + 16) * 2.0 ** -24 * (dz.abs() + each)))
        dbr += dz.sum(0)
        dbb += (off + (M + 16) * 2.0 ** -24 * dz.abs()).sum(0)
        wt = wd.t().contiguous()
        _near("dx", dx[p], dz @ wt, (each + (N + 16) * 2.0 ** -24 * (dz.abs() + each)) @ wt.abs())
    _near("dw", dw, *sums)
    _near("db", db, dbr, dbb)
