"""What the autograd functions share: gradients of the first order, and tensors as the library takes them."""
import functools

import torch
from torch.autograd.function import once_differentiable

from . import fbl as _f


def first_order(backward):
    """A backward in the library's kernels, of which autograd knows no derivative: its gradients under
    create_graph may be read, but differentiating them raises.  once_differentiable marks them so only where an
    incoming gradient requires grad; without one (the gradient of a weighted sum) they would count as
    constants, though they depend on what the forward saved, and a penalty on them would drop out unseen."""
    once = once_differentiable(backward)

    @functools.wraps(backward)
    def marked(ctx, *grads):
        if not torch.is_grad_enabled():
            return backward(ctx, *grads)
        return once(ctx, *(g if g is None or g.requires_grad else g.detach().requires_grad_() for g in grads))
    return marked


def unit(t, what: str):
    """The incoming gradient as it is, if its rows have unit inner stride."""
    if t.dim() == 0 or t.stride(-1) != 1:
        raise _f.FblError(_f.FBL_ERR_LAYOUT, f"{what}: the incoming gradient needs unit inner stride, got strides "
                                             f"{tuple(t.stride())}; pass a contiguous gradient")
    return t


def matrix_of(t, what: str):
    """[..., N] as a matrix of rows: itself, or a view."""
    if t.dim() == 2:
        return t
    try:
        return t.view(-1, t.shape[-1])
    except RuntimeError as e:
        raise _f.FblError(_f.FBL_ERR_LAYOUT, f"{what}: the rows are not one strided matrix ({e}); pass it "
                                             f"contiguous") from None


def rows_of(x, width):
    """A new [..., width] tensor beside x [..., K], and it as a matrix of rows for the library to write.  (A function
    that returned a view of the matrix would have an output that torch lets nobody change in place.)"""
    out = torch.empty((*x.shape[:-1], width), dtype=x.dtype, device=x.device)
    return out, out if out.dim() == 2 else out.view(-1, width)
