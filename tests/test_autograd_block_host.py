"""The rotary and gated autograd functions as torch sees them: what may be differentiated and what may be changed in place,
and what clipping does to a parameter list (CPU).  The library's calls are replaced by stand-ins of the same shapes."""
import types

import pytest
import torch

from paper_2607_21624_amd import autograd as ag
from paper_2607_21624_amd import autograd_block as blk
from paper_2607_21624_amd import fbl as F


def _stand_ins():
    def qk_norm_rotary_fwd(q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps, q_out=None, k_out=None):
        a, b = q * 2, None if k is None else k * 2
        return (a if q_out is None else q_out.copy_(a)), (b if k_out is None else k_out.copy_(b))

    def qk_norm_rotary_bwd(gq, gk, q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps, dq=None, dk=None,
                           need_weights=True):
        a, b = gq * 2, None if gk is None else gk * 2
        w = lambda t: torch.ones_like(t) if need_weights and t is not None else None
        return (a if dq is None else dq.copy_(a)), (b if dk is None else dk.copy_(b)), w(q_weight), w(k_weight)

    def attn_fwd(q, k, v, Hq, Hkv, scale, causal):
        return q.clone(), torch.zeros(q.shape[0], Hq, q.shape[1])

    def attn_bwd(q, k, v, o, do, lse, Hq, Hkv, scale, causal, dq=None, dk=None, dv=None):
        return dq.copy_(do * q), dk.copy_(do * k), dv.copy_(do * v)

    def gated_fwd(x, w, bias, act, factors=None):
        z = x @ w
        if factors is not None:
            factors.copy_(z)
        return z[:, :w.shape[1] // 2].clone()

    def gated_bwd(dy, w_down, factors, dz=None, need_bias=True):
        dh = dy @ w_down.t()
        got = torch.cat([dh, dh], 1) * factors
        return got if dz is None else dz.copy_(got), got.sum(0) if need_bias else None

    def linear_fwd(x, w, bias=None, act="none", residual=None, out=None, z=None):
        y = x @ w if residual is None else x @ w + residual
        return y if out is None else out.copy_(y)

    def linear_bwd(dy, x, w, need_dx=True, need_dw=True, need_bias=True):
        return dy @ w.t() if need_dx else None, x.t() @ dy if need_dw else None, dy.sum(0) if need_bias else None

    def clip_grad_norm(grads, limit):
        for g in grads:
            g.data.mul_(0.5)
        return torch.tensor(float(len(grads)))

    made = {k: v for k, v in locals().items() if callable(v)}
    assert all(hasattr(F, k) for k in made)
    return types.SimpleNamespace(FblError=F.FblError, FBL_ERR_SHAPE=F.FBL_ERR_SHAPE, FBL_ERR_LAYOUT=F.FBL_ERR_LAYOUT, **made)


@pytest.fixture(autouse=True)
def library(monkeypatch):
    monkeypatch.setattr(blk, "_f", _stand_ins())


B, S, K, N = 2, 3, 8, 12
TURNS = torch.zeros(2, dtype=torch.int64)
FUNCTIONS = {
    "attention_packed_rotary": (lambda p, a, b: ag.attention_packed(p, 1, 1, turns=TURNS, q_weight=a, k_weight=b, eps=1e-6),
                                [(B, S, 3 * K), (K,), (K,)]),
    "qk_norm_rotary": (lambda q, k, a, b: sum(ag.qk_norm_rotary(q, k, 1, 1, TURNS, q_weight=a, k_weight=b, eps=1e-6)),
                       [(B, S, K), (B, S, K), (K,), (K,)]),
    "qk_norm_rotary_q": (lambda q: ag.qk_norm_rotary(q, None, 1, 0, TURNS)[0], [(B, S, K)]),
    "gated_mlp": (ag.gated_mlp, [(B, S, K), (K, 2 * N), (2 * N,), (N, K), (K,)]),
    "gated_mlp_residual": (lambda x, w1, w2, r: ag.gated_mlp(x, w1, None, w2, None, residual=r),
                           [(B, S, K), (K, 2 * N), (N, K), (B, S, K)]),
}


def test_every_function_is_here():
    known = {c for c in vars(blk).values() if isinstance(c, type) and issubclass(c, torch.autograd.Function)}
    assert len(known) == 3


@pytest.mark.parametrize("constant", [True, False])
@pytest.mark.parametrize("name", FUNCTIONS)
def test_second_derivatives_are_refused(name, constant):
    f, shapes = FUNCTIONS[name]
    leaves = [torch.randn(*s, requires_grad=True) for s in shapes]
    out = f(*leaves)
    weight = torch.ones_like(out) if constant else torch.ones_like(out).requires_grad_()
    want = torch.autograd.grad(out, leaves, weight.detach(), retain_graph=True)
    assert not any(g.requires_grad for g in want)
    got = torch.autograd.grad(out, leaves, weight, create_graph=True)
    for a, b in zip(got, want):
        assert torch.equal(a.detach(), b)
        with pytest.raises(RuntimeError, match="once_differentiable"):
            (a * a).sum().backward(retain_graph=True)


@pytest.mark.parametrize("name", [n for n in FUNCTIONS if "attention" not in n])  # attention's backward reads its output
def test_results_may_be_changed_in_place(name):
    f, shapes = FUNCTIONS[name]
    leaves = [torch.randn(*s, requires_grad=True) for s in shapes]
    out = f(*leaves)
    want = torch.autograd.grad(out, leaves, torch.ones_like(out) / 2)
    out = f(*leaves)
    assert not out._is_view()
    out /= 2
    for a, b in zip(torch.autograd.grad(out, leaves, torch.ones_like(out)), want):
        assert torch.equal(a, b)


def test_a_result_that_nothing_depends_on():
    q, k = (torch.randn(B, S, K, requires_grad=True) for _ in range(2))
    yq, yk = ag.qk_norm_rotary(q, k, 1, 1, TURNS)
    dq, dk = torch.autograd.grad(yk, (q, k), torch.ones_like(yk))
    assert torch.all(dq == 0) and torch.all(dk == 2)
    y, none = ag.qk_norm_rotary(q, None, 1, 0, TURNS)
    assert none is None
    (g,) = torch.autograd.grad(y, q, torch.ones_like(y), create_graph=True)
    assert g.requires_grad


def test_broadcast_gradients_are_refused():
    f, shapes = FUNCTIONS["gated_mlp"]
    leaves = [torch.randn(*s, requires_grad=True) for s in shapes]
    with pytest.raises(F.FblError):
        f(*leaves).sum().backward()


def test_wide_rows():
    """Rows of bf16 on the channels' stride begin further apart; others, and what would pass the products' limit, as they are."""
    like = torch.empty(0, dtype=torch.bfloat16)
    t = blk._wide(3, 16384, like)
    assert t.shape == (3, 16384) and t.stride() == (16640, 1)
    for rows, width, x in ((3, 16384 + 8, like), (3, 8192, like), (3, 16384, torch.empty(0))):
        assert blk._wide(rows, width, x).is_contiguous()
    meta = torch.empty(0, dtype=torch.bfloat16, device="meta")
    assert blk._wide((1 << 31) // 32768 - 1, 16384, meta).is_contiguous()
    assert not blk._wide((1 << 31) // 33280 - 1, 16384, meta).is_contiguous()


def test_clipping_takes_the_parameters_that_have_gradients():
    ps = [torch.zeros(3, requires_grad=True) for _ in range(3)]
    ps[0].grad, ps[2].grad = torch.ones(3), torch.ones(3)
    versions = [ps[i].grad._version for i in (0, 2)]
    assert float(ag.clip_grad_norm_((p for p in ps), 1.0)) == 2
    assert torch.all(ps[0].grad == 0.5) and ps[1].grad is None
    assert all(ps[i].grad._version > v for i, v in zip((0, 2), versions))
    assert float(ag.clip_grad_norm_(ps[0], 1.0)) == 1


@pytest.mark.parametrize("enabled", [True, False])
def test_factors_are_kept_for_a_backward_alone(monkeypatch, enabled):
    kept = []
    plain = blk._f.gated_fwd
    monkeypatch.setattr(blk._f, "gated_fwd", lambda *a, factors=None: (kept.append(factors), plain(*a, factors=factors))[1])
    w1, w2 = torch.ones(8, 32, requires_grad=True), torch.ones(16, 8)
    with torch.set_grad_enabled(enabled):
        ag.gated_mlp(torch.ones(2, 3, 8), w1, None, w2, None)
    assert len(kept) == 1 and (kept[0] is not None) == enabled
