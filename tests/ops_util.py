"""Helpers of the tests of layer norm, linear layers and the losses: elementwise
comparison with the float64 oracle."""
import numpy as np
import torch

from parity_util import note, to_np  # noqa: F401

# half a rounding step, relative: what one rounding to the storage type costs
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounded(rng, shape, dt, scale=1.0, shift=0.0):
    """(device tensor of the storage type, its values in float64)."""
    t = torch.from_numpy(np.asarray(rng.standard_normal(shape) * scale + shift, dtype=np.float32)).to(dt)
    return t.cuda(), t.double().numpy()


def check(name, got, ref, bound, halves=1.0):
    """|got - ref| <= halves * HALF * |ref| + bound, element by element (bound: what the
    fp32 sums before the rounding may be off by)."""
    g = to_np(got)
    assert g.shape == ref.shape, (name, g.shape, ref.shape)
    off = np.abs(g - ref) - halves * HALF[got.dtype] * np.abs(ref) - bound
    worst = np.unravel_index(np.argmax(np.where(np.isnan(off), np.inf, off)), off.shape) if off.size else ()
    assert np.all(off <= 0), f"{name}: {g[worst]} against {ref[worst]} at {worst}, off by {off[worst]} more than allowed"


def padded(t, extra=5, fill=float("nan")):
    """The same matrix as a view with `extra` more elements between its rows, and the buffer."""
    buf = torch.full((t.shape[0] + 1, t.shape[1] + extra), fill, dtype=t.dtype, device=t.device)
    view = buf[:-1, :t.shape[1]]
    view.copy_(t)
    return view, buf
