"""The autograd functions of a block with rotary positions and a gated feed-forward part, and the end of its step; users
have them from the autograd module, whose description names them."""
import torch

from . import fbl as _f
from .autograd_common import first_order, matrix_of, rows_of, unit


class _AttentionPackedRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, qkv, Hq, Hkv, scale, causal, turns, positions, axes, neighbours, q_weight, k_weight, eps):
        q, k, v = _packed_views(qkv, Hq, Hkv, "attention_packed")
        qk = torch.empty((*qkv.shape[:2], q.shape[2] + k.shape[2]), dtype=qkv.dtype, device=qkv.device)
        qr, kr = qk[..., :q.shape[2]], qk[..., q.shape[2]:]
        _f.qk_norm_rotary_fwd(q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps, qr, kr)
        o, lse = _f.attn_fwd(qr, kr, v, Hq, Hkv, scale, causal)
        ctx.save_for_backward(qkv, qk, o, lse, turns, positions, q_weight, k_weight)
        ctx.cfg = (Hq, Hkv, scale, causal, axes, neighbours, eps)
        return o

    @staticmethod
    @first_order
    def backward(ctx, do):
        qkv, qk, o, lse, turns, positions, q_weight, k_weight = ctx.saved_tensors
        Hq, Hkv, scale, causal, axes, neighbours, eps = ctx.cfg
        q, k, v = _packed_views(qkv, Hq, Hkv, "attention_packed")
        dqkv = torch.empty(qkv.shape, dtype=qkv.dtype, device=qkv.device)
        dq, dk, dv = _packed_views(dqkv, Hq, Hkv, "attention_packed")
        _f.attn_bwd(qk[..., :q.shape[2]], qk[..., q.shape[2]:], v, o, unit(do, "attention_packed"), lse, Hq, Hkv, scale, causal,
                    dq=dq, dk=dk, dv=dv)
        # the gradients of what attention read become those of the projection where they lie
        need = ctx.needs_input_grad[9] or ctx.needs_input_grad[10]
        _, _, dqw, dkw = _f.qk_norm_rotary_bwd(dq, dk, q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight,
                                               eps, dq=dq, dk=dk, need_weights=need)
        return (dqkv,) + (None,) * 8 + (dqw, dkw, None)


def _tuple(axes):
    return None if axes is None else tuple(axes)  # kept for the backward, whatever becomes of the caller's list


def _packed_views(qkv, Hq: int, Hkv: int, where: str):
    """Q, K and V in a packed [B, S, (Hq + 2 Hkv) d] tensor."""
    if qkv.dim() != 3 or qkv.shape[2] % (Hq + 2 * Hkv):
        raise _f.FblError(_f.FBL_ERR_SHAPE, f"{where}: qkv has shape {tuple(qkv.shape)}, needs [B, S, ({Hq} + 2 * {Hkv}) d]")
    d = qkv.shape[2] // (Hq + 2 * Hkv)
    return qkv[..., :Hq * d], qkv[..., Hq * d:(Hq + Hkv) * d], qkv[..., (Hq + Hkv) * d:]


def attention_packed_rotary(qkv, Hq, Hkv, scale, causal, turns, positions, axes, neighbours, q_weight, k_weight, eps):
    """autograd.attention_packed where there is something to turn or to norm."""
    return _AttentionPackedRotary.apply(qkv, Hq, Hkv, scale, causal, turns, positions, _tuple(axes), neighbours, q_weight,
                                        k_weight, eps)


class _QkNormRotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps):
        y = _f.qk_norm_rotary_fwd(q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight, k_weight, eps)
        ctx.save_for_backward(q if eps is not None else None, k if eps is not None else None, turns, positions, q_weight,
                              k_weight)
        ctx.cfg = (Hq, Hkv, axes, neighbours, eps)
        return y

    @staticmethod
    @first_order
    def backward(ctx, gq, gk):
        q, k, turns, positions, q_weight, k_weight = ctx.saved_tensors
        Hq, Hkv, axes, neighbours, eps = ctx.cfg
        gq, gk = unit(gq, "qk_norm_rotary"), None if gk is None else unit(gk, "qk_norm_rotary")
        need = ctx.needs_input_grad[8] or ctx.needs_input_grad[9]
        dq, dk, dqw, dkw = _f.qk_norm_rotary_bwd(gq, gk, q, k, Hq, Hkv, turns, positions, axes, neighbours, q_weight,
                                                 k_weight, eps, need_weights=need)
        return dq, dk, None, None, None, None, None, None, dqw, dkw, None


def qk_norm_rotary(q, k, Hq: int, Hkv: int, turns=None, positions=None, axes=None, neighbours: bool = False, q_weight=None,
                   k_weight=None, eps=None):
    return _QkNormRotary.apply(q, k, Hq, Hkv, turns, positions, _tuple(axes), bool(neighbours), q_weight, k_weight, eps)


def _wide(rows: int, width: int, like):
    """A new matrix for a kernel's intermediate.  Rows of bfloat16 that are 32 KB or more and a multiple of 1 KB begin 512
    bytes further apart: a product that walks down them (dx takes 256 rows of dz a tile) would else meet few of the
    memory's channels (gated step of 4096 tokens, 2048 -> 8192 1233 -> 1181 us, 4096 -> 11008 3112 -> 3085; rows of 16 KB gain
    nothing, 8192 tokens 1024 -> 4096 705 -> 722)."""
    row = 2 * width
    if like.dtype != torch.bfloat16 or row < 1 << 15 or row % 1024 or rows * (row + 512) >= 1 << 31:  # (the products' limit)
        return like.new_empty((rows, width))
    return like.new_empty((rows, width + 256))[:, :width]


class _GatedMlp(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w1, b1, w2, b2, residual, act, grads):
        x2 = matrix_of(x, "gated_mlp")
        res2 = None
        if residual is not None:
            if residual.shape != (*x.shape[:-1], w2.shape[1]):
                raise _f.FblError(_f.FBL_ERR_SHAPE, f"gated_mlp: residual has shape {tuple(residual.shape)}, needs "
                                                    f"{(*x.shape[:-1], w2.shape[1])}")
            res2 = matrix_of(residual, "gated_mlp: residual")
        factors = None
        if grads and any(ctx.needs_input_grad[:3]):
            factors = _wide(x2.shape[0], w1.shape[1], x)
        h = _f.gated_fwd(x2, w1, b1, act, factors=factors)
        if x.dim() == 2:
            y = _f.linear_fwd(h, w2, b2, residual=res2)
        else:
            y, y2 = rows_of(x, w2.shape[1])
            _f.linear_fwd(h, w2, b2, residual=res2, out=y2)
        ctx.save_for_backward(x2, w1, w2, factors, h)
        ctx.xshape = x.shape
        return y

    @staticmethod
    @first_order
    def backward(ctx, dy):
        x2, w1, w2, factors, h = ctx.saved_tensors
        need = ctx.needs_input_grad
        dx = dw1 = db1 = dw2 = db2 = None
        if any(need[:5]):
            dy2 = matrix_of(unit(dy, "gated_mlp"), "gated_mlp: the incoming gradient")
            if any(need[:3]):
                wide = None if factors.is_contiguous() else _wide(*factors.shape, factors)
                dz, db1 = _f.gated_bwd(dy2, w2, factors, dz=wide, need_bias=need[2])
                if need[0] or need[1]:
                    dx, dw1, _ = _f.linear_bwd(dz, x2, w1, need_dx=need[0], need_dw=need[1], need_bias=False)
            if need[3] or need[4]:
                _, dw2, db2 = _f.linear_bwd(dy2, h, w2, need_dx=False, need_dw=need[3], need_bias=need[4])
        if dx is not None and len(ctx.xshape) != 2:
            dx = dx.view(ctx.xshape)
        return dx, dw1, db1, dw2, db2, dy if need[5] else None, None, None


def gated_mlp(x, w1, b1, w2, b2, act: str = "silu", residual=None):
    # under no_grad needs_input_grad still tells of the parameters: nothing is kept there
    return _GatedMlp.apply(x, w1, b1, w2, b2, residual, act, torch.is_grad_enabled())


def clip_grad_norm_(parameters, limit: float):
    grads = [p.grad for p in ([parameters] if isinstance(parameters, torch.Tensor) else parameters) if p.grad is not None]
    norm = _f.clip_grad_norm(grads, limit)
    torch.autograd.graph.increment_version(grads)  # changed in place
    return norm
