"""torch.autograd wrappers over the C ABI: attention, linear layers, layer norm and
the losses of a linear head, usable inside an ordinary training step.  Argument
marshalling only -- every forward and backward runs in the library's kernels;
torch provides the tensors, the stream and the autograd graph.

  attention(q, k, v, Hq, Hkv, scale=None, causal=False, kv_len=None) -> O
      q [B, S_q, Hq*d], k and v [B, S_kv, Hkv*d], token-major (any row
      stride, inner stride 1); gradients flow to q, k and v.
  attention_packed(qkv, Hq, Hkv, scale=None, causal=False) -> O
      qkv [B, S, (Hq + 2 Hkv) d], the packed output of a fused QKV
      projection; its gradient is one packed tensor of the same shape.
  linear(x, w, bias=None, act="none", residual=None) -> act(x @ w + bias) + residual
      x [..., K] (rows contiguous), w [K, N]; gradients x and w by the data-
      and weight-gradient products, no transposed copy of either.  bias [N],
      act "none", "relu", "gelu", "gelu_tanh" or "silu", residual [..., N].
  mlp(x, w1, b1, w2, b2, act="gelu", residual=None) -> act(x @ w1 + b1) @ w2 + b2 + residual
      a block's feed-forward part; its backward takes the activation's
      derivative and b1's gradient in the epilogue of the data gradient.  b1, b2 may be None.
  layer_norm(x, weight=None, bias=None, eps=1e-5) -> y
      x [..., N] (rows one strided matrix), weight and bias [N]; gradients to all three.
  linear_cross_entropy(x, w, labels, ignore_index=-100, reduction="mean") -> loss
      softmax cross entropy of the logits x @ w over a vocabulary, which are never kept:
      x [..., K], w [K, V] (or table.t() of a [V, K] table), labels [...]
      int64; gradients to x and w.  loss float32: the mean over the rows not
      labelled ignore_index, their "sum", or every row's ("none", [...]).
  linear_distillation(x, w, index, logits, temperature=1.0, reduction="mean") -> loss
      the same from a teacher's top logits: index int64 and logits [..., top].  The
      teacher is a constant: logits that require grad get no gradient from here.

Gradients are those of the first order: taken with create_graph they hold their
values, and differentiating them raises an error.

The incoming gradient is read in place, never copied: it must have unit
inner stride (any row stride from the width on), like every tensor the kernels read.  Autograd
can hand over a broadcast view (the gradient of a plain .sum(), inner stride
0); such a gradient is rejected with FblError, and the caller makes it
contiguous (or backpropagates a materialised tensor) instead.

Capturing a backward pass into a graph: run a step on the capturing stream first and
let go of every eager loss or output of the same leaves.  While one lives, torch
keeps the leaves' accumulation on that graph's stream, and a capture that meets another
stream ends with an error or the process.
"""
import functools
import math

import torch
from torch.autograd.function import once_differentiable

from . import fbl as _f


def _first_order(backward):
    """A backward in the library's kernels, of which autograd knows no derivative: its gradients under
    create_graph may be read, but differentiating them raises.  once_differentiable marks them so only where an
    incoming gradient requires grad; without one (the gradient of a weighted sum) they would count as
    constants, though they depend on what the forward saved, and a penalty on them would drop out unseen."""
    once = once_differentiable(backward)

    @functools.wraps(backward)
    def marked(ctx, *grads):
        if torch.is_grad_enabled():
            grads = tuple(g if g.requires_grad else g.detach().requires_grad_() for g in grads)
        return once(ctx, *grads)
    return marked


def _unit(t, what: str):
    """The incoming gradient as it is, if its rows have unit inner stride."""
    if t.dim() == 0 or t.stride(-1) != 1:
        raise _f.FblError(_f.FBL_ERR_LAYOUT, f"{what}: the incoming gradient needs unit inner stride, got strides "
                                             f"{tuple(t.stride())}; pass a contiguous gradient")
    return t


def _matrix_of(t, what: str):
    """[..., N] as a matrix of rows, a view."""
    try:
        return t.view(-1, t.shape[-1])
    except RuntimeError as e:
        raise _f.FblError(_f.FBL_ERR_LAYOUT, f"{what}: the rows are not one strided matrix ({e}); pass it "
                                             f"contiguous") from None


def _rows_of(x, width):
    """A new [..., width] tensor beside x [..., K], and it as a matrix of rows for the library to write.  (A function
    that returned a view of the matrix would have an output that torch lets nobody change in place.)"""
    out = torch.empty((*x.shape[:-1], width), dtype=x.dtype, device=x.device)
    return out, out if out.dim() == 2 else out.view(-1, width)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, Hq, Hkv, scale, causal, kv_len):
        o, lse = _f.attn_fwd(q, k, v, Hq, Hkv, scale, causal, kv_len)
        ctx.save_for_backward(q, k, v, o, lse, kv_len if kv_len is not None else torch.empty(0))
        ctx.cfg = (Hq, Hkv, scale, causal, kv_len is not None)
        return o

    @staticmethod
    @_first_order
    def backward(ctx, do):
        q, k, v, o, lse, kv = ctx.saved_tensors
        Hq, Hkv, scale, causal, has_kv = ctx.cfg
        dq, dk, dv = _f.attn_bwd(q, k, v, o, _unit(do, 'attention'), lse, Hq, Hkv, scale, causal,
                                 kv if has_kv else None)
        return dq, dk, dv, None, None, None, None, None


def attention(q, k, v, Hq: int, Hkv: int, scale=None, causal: bool = False, kv_len=None):
    if scale is None:
        scale = 1.0 / math.sqrt(q.shape[-1] // Hq)
    return _Attention.apply(q, k, v, Hq, Hkv, float(scale), bool(causal), kv_len)


class _AttentionPacked(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, Hq, Hkv, scale, causal):
        o, lse = _f.attn_fwd_packed(qkv, Hq, Hkv, scale, causal)
        ctx.save_for_backward(qkv, o, lse)
        ctx.cfg = (Hq, Hkv, scale, causal)
        return o

    @staticmethod
    @_first_order
    def backward(ctx, do):
        qkv, o, lse = ctx.saved_tensors
        Hq, Hkv, scale, causal = ctx.cfg
        dqkv = _f.attn_bwd_packed(qkv, o, _unit(do, 'attention_packed'), lse, Hq, Hkv, scale, causal)
        return dqkv, None, None, None, None


def attention_packed(qkv, Hq: int, Hkv: int, scale=None, causal: bool = False):
    if scale is None:
        scale = 1.0 / math.sqrt(qkv.shape[-1] // (Hq + 2 * Hkv))
    return _AttentionPacked.apply(qkv, Hq, Hkv, float(scale), bool(causal))


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w):
        x2 = x.reshape(-1, x.shape[-1])  # a view for token-major activations
        y, y2 = _rows_of(x, w.shape[-1])
        _f.proj(_f.FBL_PROJ_FWD, x2, w, out=y2)
        ctx.save_for_backward(x2, w)
        ctx.xshape = x.shape
        return y

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x2, w = ctx.saved_tensors
        dy = _unit(dy, "linear")
        try:
            dy2 = dy.view(-1, dy.shape[-1])  # a view: token rows of the incoming gradient
        except RuntimeError as e:
            raise _f.FblError(_f.FBL_ERR_LAYOUT, f"linear: the incoming gradient's rows are not one strided "
                                                 f"matrix ({e}); pass a contiguous gradient") from None
        dx = dw = None
        if ctx.needs_input_grad[0]:
            dx = _f.proj(_f.FBL_PROJ_BWD_DATA, dy2, w).view(ctx.xshape)
        if ctx.needs_input_grad[1]:
            dw = _f.proj(_f.FBL_PROJ_BWD_WEIGHT, x2, dy2)
        return dx, dw


class _LinearAct(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, residual, act):
        x2 = _matrix_of(x, "linear")
        N = w.shape[1]
        res2 = None
        if residual is not None:
            if residual.shape != (*x.shape[:-1], N):
                raise _f.FblError(_f.FBL_ERR_SHAPE, f"linear: residual has shape {tuple(residual.shape)}, needs "
                                                    f"{(*x.shape[:-1], N)}")
            res2 = _matrix_of(residual, "linear: residual")
        z = None
        if act != "none" and any(ctx.needs_input_grad[:3]):
            z = torch.empty((x2.shape[0], N), dtype=x.dtype, device=x.device)
        y, y2 = _rows_of(x, N)
        _f.linear_fwd(x2, w, bias, act, res2, out=y2, z=z)
        ctx.save_for_backward(x2, w, z)
        ctx.cfg = (x.shape, act)
        return y

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x2, w, z = ctx.saved_tensors
        xshape, act = ctx.cfg
        need = ctx.needs_input_grad
        dx = dw = db = None
        if any(need[:3]):
            dy2 = _matrix_of(_unit(dy, "linear"), "linear: the incoming gradient")
            dx, dw, db = _f.linear_bwd(dy2, x2, w, z, act, need_dx=need[0], need_dw=need[1], need_bias=need[2])
        return dx.view(xshape) if need[0] else None, dw, db, dy if need[3] else None, None


def linear(x, w, bias=None, act: str = "none", residual=None):
    if bias is None and act == "none" and residual is None:
        return _Linear.apply(x, w)
    return _LinearAct.apply(x, w, bias, residual, act)


class _Mlp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, residual, act):
        x2 = _matrix_of(x, "mlp")
        res2 = None
        if residual is not None:
            if residual.shape != (*x.shape[:-1], w2.shape[1]):
                raise _f.FblError(_f.FBL_ERR_SHAPE, f"mlp: residual has shape {tuple(residual.shape)}, needs "
                                                    f"{(*x.shape[:-1], w2.shape[1])}")
            res2 = _matrix_of(residual, "mlp: residual")
        z = None
        if act != "none" and any(ctx.needs_input_grad[:3]):
            z = torch.empty((x2.shape[0], w1.shape[1]), dtype=x.dtype, device=x.device)
        h = _f.linear_fwd(x2, w1, b1, act, z=z)
        y, y2 = _rows_of(x, w2.shape[1])
        _f.linear_fwd(h, w2, b2, residual=res2, out=y2)
        ctx.save_for_backward(x2, w1, w2, z, h)
        ctx.cfg = (x.shape, act)
        return y

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x2, w1, w2, z, h = ctx.saved_tensors
        xshape, act = ctx.cfg
        need = ctx.needs_input_grad
        first, second = any(need[:3]), need[3] or need[4]
        dx = dw1 = db1 = dw2 = db2 = None
        if first or second:
            dy2 = _matrix_of(_unit(dy, "mlp"), "mlp: the incoming gradient")
            # the hidden layer's gradient arrives as that of its pre-activation
            db1 = torch.empty(w1.shape[1], dtype=w1.dtype, device=w1.device) if need[2] else None
            dz, dw2, db2 = _f.linear_bwd(dy2, h, w2, need_dx=first, need_dw=need[3], need_bias=need[4],
                                         x_act=act if first else "none", x_z=z if first else None, dxbias=db1)
            if need[0] or need[1]:
                dx, dw1, _ = _f.linear_bwd(dz, x2, w1, need_dx=need[0], need_dw=need[1], need_bias=False)
        return dx.view(xshape) if need[0] else None, dw1, db1, dw2, db2, dy if need[5] else None, None


def mlp(x, w1, b1, w2, b2, act: str = "gelu", residual=None):
    return _Mlp.apply(x, w1, b1, w2, b2, residual, act)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps):
        x2 = _matrix_of(x, "layer_norm")
        y, y2 = _rows_of(x, x.shape[-1])
        _, mean, rstd = _f.layer_norm_fwd(x2, weight, bias, eps, out=y2)
        ctx.save_for_backward(x2, mean, rstd, weight)
        ctx.xshape = x.shape
        return y

    @staticmethod
    @_first_order
    def backward(ctx, dy):
        x2, mean, rstd, weight = ctx.saved_tensors
        dy2 = _matrix_of(_unit(dy, "layer_norm"), "layer_norm: the incoming gradient")
        dx, dw, db = _f.layer_norm_bwd(dy2, x2, mean, rstd, weight, need_weight=ctx.needs_input_grad[1],
                                       need_bias=ctx.needs_input_grad[2])
        return dx.view(ctx.xshape), dw, db, None


def layer_norm(x, weight=None, bias=None, eps: float = 1e-5):
    return _LayerNorm.apply(x, weight, bias, float(eps))


def _reduction(reduction, where: str):
    if reduction not in ("mean", "sum", "none"):
        raise _f.FblError(_f.FBL_ERR_ARG, f"{where}: reduction {reduction!r}, there are mean, sum and none")


def _reduced(x, reduction):
    """The loss to return, a tensor of its own that may be changed in place, and the argument by which the library
    writes it: the mean, the first number of total (in whose memory the sum stands), or every row's."""
    new = functools.partial(torch.empty, dtype=torch.float32, device=x.device)
    if reduction == "mean":
        mean = new(())
        return mean, {"mean": mean}
    if reduction == "sum":
        total = new(2)
        return new(0).set_(total.untyped_storage(), 0, (), ()), {"total": total}
    loss = new(x.shape[:-1])
    return loss, {"loss": loss.view(-1)}


def _loss_grad(dloss, reduction, M: int):
    """The incoming gradient as the library takes it: one number, or one for each row (a broadcast
    one included)."""
    if reduction != "none":
        return dloss
    return dloss.reshape(M)


class _LinearCrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, labels, ignore_index, reduction):
        where = "linear_cross_entropy"
        _reduction(reduction, where)
        x2 = _matrix_of(x, where)
        if labels.shape != x.shape[:-1]:
            raise _f.FblError(_f.FBL_ERR_SHAPE, f"{where}: labels have shape {tuple(labels.shape)}, need "
                                                f"{tuple(x.shape[:-1])}")
        labels2 = labels.reshape(-1).contiguous()
        result, out = _reduced(x, reduction)
        _, lse, total = _f.linear_ce_fwd(x2, w, labels2, ignore_index, **out)
        ctx.save_for_backward(x2, w, labels2, lse, total if reduction == "mean" else None)
        ctx.cfg = (x.shape, ignore_index, reduction)
        return result

    @staticmethod
    @_first_order
    def backward(ctx, dloss):
        x2, w, labels, lse, total = ctx.saved_tensors
        xshape, ignore_index, reduction = ctx.cfg
        need = ctx.needs_input_grad
        dx, dw = _f.linear_ce_bwd(_loss_grad(dloss, reduction, x2.shape[0]), x2, w, labels, lse, total, ignore_index,
                                  need_dx=need[0], need_dw=need[1])
        return dx.view(xshape) if need[0] else None, dw, None, None, None


def linear_cross_entropy(x, w, labels, ignore_index: int = -100, reduction: str = "mean"):
    return _LinearCrossEntropy.apply(x, w, labels, int(ignore_index), reduction)


class _LinearDistillation(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, index, logits, temperature, reduction):
        where = "linear_distillation"
        _reduction(reduction, where)
        x2 = _matrix_of(x, where)
        if index.shape[:-1] != x.shape[:-1] or logits.shape != index.shape:
            raise _f.FblError(_f.FBL_ERR_SHAPE, f"{where}: index {tuple(index.shape)} and logits {tuple(logits.shape)} need "
                                                f"the shape {tuple(x.shape[:-1])} + (top,)")
        index2, logits2 = _matrix_of(index, where), _matrix_of(logits, where)
        result, out = _reduced(x, reduction)
        _, lse, prob, total = _f.linear_kd_fwd(x2, w, index2, logits2, temperature, **out)
        ctx.save_for_backward(x2, w, index2, prob, lse, total if reduction == "mean" else None)
        ctx.cfg = (x.shape, temperature, reduction)
        return result

    @staticmethod
    @_first_order
    def backward(ctx, dloss):
        x2, w, index, prob, lse, total = ctx.saved_tensors
        xshape, temperature, reduction = ctx.cfg
        need = ctx.needs_input_grad
        dx, dw = _f.linear_kd_bwd(_loss_grad(dloss, reduction, x2.shape[0]), x2, w, index, prob, lse, temperature, total,
                                  need_dx=need[0], need_dw=need[1])
        return dx.view(xshape) if need[0] else None, dw, None, None, None, None


def linear_distillation(x, w, index, logits, temperature: float = 1.0, reduction: str = "mean"):
    return _LinearDistillation.apply(x, w, index, logits, float(temperature), reduction)
