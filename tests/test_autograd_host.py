"""The autograd functions as torch sees them: what may be differentiated and what may be changed in place (CPU).
The library's calls are replaced by stand-ins of the same shapes, whose values are of no account here."""
import types

import pytest
import torch

from paper_2607_21624_amd import autograd as ag
from paper_2607_21624_amd import fbl as F


def _into(out, shape, dtype, value):
    """The caller's tensor or a new one, filled with `value`."""
    out = torch.empty(shape, dtype=dtype) if out is None else out
    assert tuple(out.shape) == tuple(shape)
    return out.fill_(value)


def _stand_ins():
    f32 = torch.float32

    def attn_fwd(q, k, v, Hq, Hkv, scale, causal, kv_len):
        return q.clone(), torch.zeros(q.shape[0], Hq, q.shape[1])

    def attn_bwd(q, k, v, o, do, lse, Hq, Hkv, scale, causal, kv_len):
        return do * q, do * k, do * v

    def attn_fwd_packed(qkv, Hq, Hkv, scale, causal):
        return qkv[..., :qkv.shape[-1] * Hq // (Hq + 2 * Hkv)].clone(), torch.zeros(qkv.shape[0], Hq, qkv.shape[1])

    def attn_bwd_packed(qkv, o, do, lse, Hq, Hkv, scale, causal):
        return torch.ones_like(qkv)

    def proj(op, a, b, out=None):
        if op == F.FBL_PROJ_FWD:
            r = a @ b
        else:
            r = a @ b.t() if op == F.FBL_PROJ_BWD_DATA else a.t() @ b
        return r if out is None else out.copy_(r)

    def linear_fwd(x, w, bias=None, act="none", residual=None, out=None, z=None):
        if z is not None:
            z.copy_(x @ w)
        r = x @ w if residual is None else x @ w + residual
        return r if out is None else out.copy_(r)

    def linear_bwd(dy, x, w, z=None, act="none", need_dx=True, need_dw=True, need_bias=True, x_act="none", x_z=None,
                   dxbias=None):
        if dxbias is not None:
            dxbias.copy_((dy @ w.t()).sum(0))
        return (dy @ w.t() if need_dx else None, x.t() @ dy if need_dw else None, dy.sum(0) if need_bias else None)

    def layer_norm_fwd(x, weight, bias, eps, out=None):
        return _into(out, x.shape, x.dtype, 1.0), torch.zeros(len(x)), torch.ones(len(x))

    def layer_norm_bwd(dy, x, mean, rstd, weight, need_weight=True, need_bias=True):
        return dy * x, dy.sum(0) if need_weight else None, dy.sum(0) if need_bias else None

    def losses(x, loss, total, mean):
        M = len(x)
        loss = _into(loss, (M,), f32, 2.0)
        total = _into(total, (2,), f32, float(M))
        total[0] *= 2
        if mean is not None:
            mean.fill_(2.0)
        return loss, torch.zeros(M), total

    def linear_ce_fwd(x, w, labels, ignore_index, loss=None, total=None, mean=None):
        assert labels.shape == (len(x),) and labels.is_contiguous()
        return losses(x, loss, total, mean)

    def grads(g, x, w, total, need_dx, need_dw):
        g = (g if g.dim() else g.expand(len(x))) / (1.0 if total is None else total[1])
        dz = g[:, None].expand(len(x), w.shape[1])
        return dz @ w.t() if need_dx else None, x.t() @ dz if need_dw else None

    def linear_ce_bwd(g, x, w, labels, lse, total, ignore_index, need_dx=True, need_dw=True):
        return grads(g, x, w, total, need_dx, need_dw)

    def linear_kd_fwd(x, w, index, logits, temperature, loss=None, total=None, mean=None):
        loss, lse, total = losses(x, loss, total, mean)
        return loss, lse, torch.zeros(index.shape), total

    def linear_kd_bwd(g, x, w, index, prob, lse, temperature, total, need_dx=True, need_dw=True):
        return grads(g, x, w, total, need_dx, need_dw)

    made = dict(locals())
    made = {k: v for k, v in made.items() if callable(v) and not k.startswith("_") and hasattr(F, k)}
    consts = {k: getattr(F, k) for k in dir(F) if k.startswith("FBL_")}
    return types.SimpleNamespace(FblError=F.FblError, **consts, **made)


@pytest.fixture(autouse=True)
def library(monkeypatch):
    monkeypatch.setattr(ag, "_f", _stand_ins())


def _randn(*shape):
    return torch.randn(*shape, requires_grad=True)


B, S, K, N, V = 2, 3, 8, 12, 10
LABELS = torch.zeros(B, S, dtype=torch.int64)
LOGITS = torch.zeros(B, S, 1)
# every autograd function: leaves -> output
FUNCTIONS = {
    "attention": (lambda q, k, v: ag.attention(q, k, v, 2, 2), [(B, S, K)] * 3),
    "attention_packed": (lambda p: ag.attention_packed(p, 1, 1), [(B, S, 3 * K)]),
    "linear": (ag.linear, [(B, S, K), (K, N)]),
    "linear_bias": (ag.linear, [(B, S, K), (K, N), (N,)]),
    "linear_residual": (lambda x, w, r: ag.linear(x, w, residual=r), [(B, S, K), (K, N), (B, S, N)]),
    "mlp": (ag.mlp, [(B, S, K), (K, N), (N,), (N, K), (K,)]),
    "layer_norm": (ag.layer_norm, [(B, S, K), (K,), (K,)]),
    **{f"linear_cross_entropy_{r}": (lambda x, w, r=r: ag.linear_cross_entropy(x, w, LABELS, reduction=r), [(B, S, K), (K, V)])
       for r in ("mean", "sum", "none")},
    **{f"linear_distillation_{r}": (lambda x, w, r=r: ag.linear_distillation(x, w, LABELS[..., None], LOGITS, 2.0, r),
                                    [(B, S, K), (K, V)]) for r in ("mean", "sum", "none")},
}


def test_every_function_is_here():
    known = {c for c in vars(ag).values() if isinstance(c, type) and issubclass(c, torch.autograd.Function)}
    assert len(known) == 8 and len({f.split("_mean")[0] for f in FUNCTIONS}) >= len(known)


@pytest.mark.parametrize("constant", [True, False])
@pytest.mark.parametrize("name", FUNCTIONS)
def test_second_derivatives_are_refused(name, constant):
    """Gradients taken with create_graph hold their values, and differentiating any of them raises, whether the
    incoming gradient is a constant (a weighted sum of the outputs) or depends on something."""
    f, shapes = FUNCTIONS[name]
    leaves = [_randn(*s) for s in shapes]
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
    """loss /= steps, or a layer's output scaled where it stands: allowed, with the gradient that goes with it."""
    f, shapes = FUNCTIONS[name]
    leaves = [_randn(*s) for s in shapes]
    for lead in (leaves, [t if t.dim() < 3 else t[0] for t in leaves]):  # [..., K] of three dimensions and of two
        if lead is not leaves and ("cross" in name or "distillation" in name):
            continue
        out = f(*lead)
        value = out.detach().clone()
        want = torch.autograd.grad(out, lead, torch.ones_like(out) / 2)
        out = f(*lead)
        assert not out._is_view()
        out /= 2
        assert torch.equal(out.detach(), value / 2)
        for a, b in zip(torch.autograd.grad(out, lead, torch.ones_like(out)), want):
            assert torch.equal(a, b)


def test_labels_of_any_strides():
    """Labels of a view are copied, whether or not they could be one strided row."""
    ids = torch.arange(B * (S + 1) * 2).view(B, S + 1, 2) % V
    for labels in (ids[:, 1:, 0], ids[:, :S, 1], ids[:1, :1, :1].expand(B, S, 1)[..., 0]):
        ag.linear_cross_entropy(torch.randn(B, S, K), torch.randn(K, V), labels)
    ag.linear_cross_entropy(torch.randn(S, K), torch.randn(K, V), ids[0, :S, 0])
