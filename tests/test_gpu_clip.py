"""The global norm of gradients and clipping by it, against float64 (GPU).

Bounds.  Squares of the storage types are exact in float64 or rounded there, and so are the sums: the norm is off by its one
rounding to fp32, half a step.  The scale is computed from that norm in float64 and rounded to fp32: half a step of the
norm's and half its own, 2^-24 each, and the product's rounding to fp32 and to the storage."""
import math

import numpy as np
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import DTYPES, HALF, note, rounded
from oracle import gated_block as oracle
from paper_2607_21624_amd import autograd as ag

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _grads(sizes, dts, seed=0, scale=1.0):
    rng = np.random.default_rng(seed)
    made = [rounded(rng, s, DTYPES[dts[i % len(dts)]], scale * (1 + i % 5)) for i, s in enumerate(sizes)]
    return [m[0] for m in made], [m[1] for m in made]


def _check(out, ref, limit, norm, got_norm):
    assert abs(float(got_norm) - norm) <= U * norm
    scale = oracle.clip_scale(norm, limit)
    for o, r in zip(out, ref):
        want = r * scale
        off = np.abs(o.double().cpu().numpy() - want)
        assert np.all(off <= (HALF[o.dtype] + 4 * U) * np.abs(want) + 2.0 ** -133), (o.dtype, o.shape)


SIZES = [(1,), (7,), (8,), (9,), (4, 5), (255, 257), (16384,), (16385,), (8192,), (8191,), (3, 16384), (1000, 331), (2, 0)]


@pytest.mark.parametrize("dts", [["f32"], ["bf16"], ["bf16", "f32"], ["f32", "bf16", "bf16"]])
@pytest.mark.parametrize("which", ["out", "in place", "separate"])
def test_lists(dts, which):
    grads, ref = _grads(SIZES, dts)
    norm = oracle.grad_norm(ref)
    note(f"clip {dts} {which}")
    for limit in (0.5 * norm, 1e-3, 2 * norm):
        mine = [g.clone() for g in grads]
        if which == "out":
            out = [torch.full_like(g, 9.0) for g in grads]
            n = fbl.clip_grad_norm(mine, limit, out=out)
            assert all(torch.equal(a, b) for a, b in zip(mine, grads))
        elif which == "in place":
            n, out = fbl.clip_grad_norm(mine, limit), mine
        else:
            n, out = fbl.grad_norm(mine), mine
            fbl.clip_grads(mine, n, limit)
        torch.cuda.synchronize()
        _check(out, ref, limit, norm, n)
        if limit > norm:
            assert all(torch.equal(a, b) for a, b in zip(out, grads))


def test_one_tensor_alone_each_size():
    for dt in DTYPES.values():
        for n in (1, 3, 4, 5, 7, 8, 9, 63, 64, 65, 2047, 2048, 2049, 8191, 8193, 16383, 16384, 16391, 40000):
            g, r = rounded(np.random.default_rng(n), (n + 3,), dt)
            buf = torch.full((n + 40,), 5.0, dtype=dt, device="cuda")
            view = buf[17:17 + n]  # begins at any element
            view.copy_(g[:n])
            norm = oracle.grad_norm([r[:n]])
            got = fbl.clip_grad_norm([view], norm / 3)
            _check([view], [r[:n]], norm / 3, norm, got)
            assert torch.all(buf[:17] == 5.0) and torch.all(buf[17 + n:] == 5.0)


def test_more_tensors_than_a_launch():
    grads, ref = _grads([(5 + i % 70, 3) for i in range(300)], ["bf16", "f32"])
    norm = oracle.grad_norm(ref)
    n = fbl.clip_grad_norm(grads, norm / 7)
    _check(grads, ref, norm / 7, norm, n)
    assert fbl.grad_norm_workspace(grads) == 3 * 1024 * 8


def test_many_chunks():
    g, _ = rounded(np.random.default_rng(1), (1 << 16,), torch.bfloat16)
    big = g.repeat(1200)  # 9600 chunks on 1024 workgroups
    want = math.sqrt(1200 * float((g.double() ** 2).sum()))
    n = fbl.grad_norm([big, g.float()])
    want = math.sqrt(want ** 2 + float((g.double() ** 2).sum()))
    assert abs(float(n) - want) <= U * want
    out = torch.empty_like(big)
    fbl.clip_grads([big], n, want / 2, out=[out])
    scale = torch.tensor(oracle.clip_scale(float(n), want / 2), dtype=torch.float32, device="cuda")
    assert torch.equal(out, (big.float() * scale).to(torch.bfloat16))


def test_large_and_small_values():
    # squares that overflow fp32, and that vanish in it
    for x, n in ((3e38, 4), (1e30, 5000), (1e-30, 5000), (2e-38, 3)):
        g = torch.full((n,), x, device="cuda")
        norm = float(g[0].double()) * math.sqrt(n)
        got = float(fbl.grad_norm([g]))
        if norm > torch.finfo(torch.float32).max:
            assert got == math.inf
        else:
            assert abs(got - norm) <= U * norm
    zero = torch.zeros(100, device="cuda")
    assert float(fbl.clip_grad_norm([zero], 1.0)) == 0 and torch.all(zero == 0)
    assert float(fbl.clip_grad_norm([zero[:0]], 1.0)) == 0


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_infinities_and_nan(bad):
    g = [torch.ones(50, device="cuda"), torch.ones(3, dtype=torch.bfloat16, device="cuda")]
    g[0][17] = bad
    n = fbl.clip_grad_norm(g, 1.0)
    if math.isnan(bad):
        assert math.isnan(float(n)) and all(torch.isnan(t).all() for t in g)
    else:  # the scale is 0
        assert float(n) == math.inf and torch.isnan(g[0][17]) and int((g[0] == 0).sum()) == 49 and torch.all(g[1] == 0)


def test_limits():
    g = [torch.full((4,), 3.0, device="cuda")]  # norm 6
    assert float(fbl.clip_grad_norm(g, math.inf)) == 6 and torch.all(g[0] == 3)
    assert float(fbl.clip_grad_norm(g, 0.0)) == 6 and torch.all(g[0] == 0)


def test_any_order_of_dimensions_and_refusals_on_the_gpu():
    x, r = rounded(np.random.default_rng(2), (40, 30), torch.float32)
    table = x.t()  # a table's gradient as a transposed view
    norm = oracle.grad_norm([r])
    n = fbl.clip_grad_norm([table], norm / 2)
    _check([x], [r], norm / 2, norm, n)
    a, b = torch.ones(8, 8, device="cuda"), torch.ones(8, 8, device="cuda")
    for grads, kw, status in (([a[:, :4]], {}, fbl.fbl.FBL_ERR_LAYOUT), ([a, a], {}, fbl.fbl.FBL_ERR_ARG),
                              ([a, a[2]], {}, fbl.fbl.FBL_ERR_ARG), ([a], dict(out=[b.t()]), fbl.fbl.FBL_ERR_SHAPE),
                              ([a], dict(out=[b.bfloat16()]), fbl.fbl.FBL_ERR_DTYPE), ([a, b], dict(out=[b, a]), fbl.fbl.FBL_ERR_ARG),
                              ([a.half()], {}, fbl.fbl.FBL_ERR_DTYPE), ([a], dict(norm=torch.zeros(2, device="cuda")), fbl.fbl.FBL_ERR_SHAPE),
                              ([a], dict(norm=a[0, 0]), fbl.fbl.FBL_ERR_ARG), ([a, b.cpu()], {}, fbl.fbl.FBL_ERR_ARG)):
        with pytest.raises(fbl.FblError) as e:
            fbl.clip_grad_norm(grads, 1.0, **kw)
        assert e.value.status == status, e.value
        assert torch.all(a == 1) and torch.all(b == 1)


def test_repeatable_workspace_and_stream():
    grads, _ = _grads([(1000, 77), (33,), (512, 512)], ["bf16", "f32"])
    n = fbl.grad_norm(grads)
    ws = torch.full((fbl.grad_norm_workspace(grads) + 64,), 0xff, dtype=torch.uint8, device="cuda")
    assert torch.equal(fbl.grad_norm(grads, workspace=ws[:-64]), n) and torch.all(ws[-64:] == 0xff)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    m = fbl.grad_norm(grads, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(m, n)
    with pytest.raises(fbl.FblError):
        fbl.grad_norm(grads, workspace=ws[:64])


def test_parameters_of_a_step():
    rng = np.random.default_rng(6)
    ps = [rounded(rng, s, torch.float32)[0].requires_grad_(True) for s in ((6, 4), (4,), (3,))]
    (ps[0] * 3).sum().backward()
    ps[1].grad = rounded(rng, (4,), torch.float32)[0]
    kept = [ps[0].grad.clone(), ps[1].grad.clone()]
    versions = [p.grad._version for p in ps[:2]]
    want = [k.double().cpu().numpy() for k in kept]
    norm = oracle.grad_norm(want)
    n = ag.clip_grad_norm_(iter(ps), norm / 4)
    _check([p.grad for p in ps[:2]], want, norm / 4, norm, n)
    assert all(p.grad._version > v for p, v in zip(ps, versions)) and ps[2].grad is None
    assert torch.equal(ag.clip_grad_norm_(ps[1], 100.0), fbl.grad_norm([ps[1].grad]))


def test_graph_replays():
    grads, _ = _grads([(300, 77), (33,), (5, 1000)], ["bf16", "f32"])
    out = [torch.empty_like(g) for g in grads]
    norm = torch.empty((), device="cuda")
    ws = torch.empty(fbl.grad_norm_workspace(grads), dtype=torch.uint8, device="cuda")
    step = lambda: fbl.clip_grad_norm(grads, 10.0, out=out, norm=norm, workspace=ws)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        grads[0].mul_(0.3)
        graph.replay()
        torch.cuda.synchronize()
        got = [norm.clone()] + [t.clone() for t in out]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, [norm] + out))


def test_offsets_past_32_bits():
    # more than 2^31 values, 2^32 bytes: a few that count at either end and around both limits
    n = (1 << 31) + 5001
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    at = torch.tensor([0, 1 << 30, (1 << 31) - 1, 1 << 31, (1 << 31) + 4097, n - 1], device="cuda")
    g[at] = torch.arange(1, 7, device="cuda").to(torch.bfloat16)  # squares add to 91
    note("clip past 32 bits")
    norm = fbl.clip_grad_norm([g], math.sqrt(91) / 2)
    assert abs(float(norm) - math.sqrt(91)) <= U * math.sqrt(91)
    scale = oracle.clip_scale(float(norm), math.sqrt(91) / 2)
    want = torch.arange(1, 7, dtype=torch.float64) * scale
    assert torch.all((g[at].double().cpu() - want).abs() <= (HALF[torch.bfloat16] + 4 * U) * want)
    g[at] = 0
    assert not torch.any(g.view(torch.int16)[: n // 2]) and not torch.any(g.view(torch.int16)[n // 2:])


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_without_a_limit_nothing_changes(bad):
    g = torch.arange(300.0, device="cuda")
    g[17] = bad
    want = g.clone()
    out = torch.zeros_like(g)
    same = lambda a: torch.equal(a.view(torch.int32), want.view(torch.int32))
    n = fbl.clip_grad_norm([g], math.inf, out=[out])
    assert same(out) and same(g) and not math.isfinite(float(n))
    fbl.clip_grad_norm([g], math.inf)
    fbl.clip_grads([g], n, math.inf)
    assert same(g)
