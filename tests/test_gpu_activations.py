"""bf16 activations and their derivatives relative to their own values, far into the negative tail (GPU).

Bounds: half a rounding step of the result, and 2^-12 of it for the arithmetic: the distribution
function's polynomial is good to 8e-5 of the tail, exp2's argument, up to 120, is rounded to 2^-18 (2e-5 of the
result with the square before it), the reciprocal and the product to 2^-22.  The derivative Phi + z phi loses what
its two terms cancel: both are below |z| phi."""
import numpy as np
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import HALF, check, note
from oracle import train as oracle

pytestmark = pytest.mark.gpu
ACTS = ("relu", "gelu", "gelu_tanh", "silu")
DT = torch.bfloat16


def _tail(z):
    """Phi(z) of negative z to its own precision."""
    from scipy.special import erfc
    return 0.5 * erfc(-z / np.sqrt(2.0))


def _refs(z, act):
    """(act, act', magnitude of the terms of act') in float64, tails included."""
    if act == "gelu":
        phi = np.exp(-0.5 * z * z) / np.sqrt(2.0 * np.pi)
        return z * _tail(z), _tail(z) + z * phi, _tail(z) + np.abs(z) * phi
    if act == "gelu_tanh":  # z s, s = 1 / (1 + exp(-2u)), the same as with the tanh
        c, a = np.sqrt(2.0 / np.pi), 0.044715
        s = 1.0 / (1.0 + np.exp(-2.0 * c * (z + a * z ** 3)))
        d = 2.0 * z * c * (1.0 + 3.0 * a * z * z) * s * (1.0 - s)
        return z * s, s + d, s + np.abs(d)
    y, g = oracle.act(z, act), oracle.act_grad(z, act)
    s = 1.0 / (1.0 + np.exp(-z))
    return y, g, np.abs(g) if act == "relu" else s + np.abs(z * s * (1.0 - s))


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [3, 200])  # a few tokens (the shared contraction below), and a tile
def test_tails(M, act):
    """z = x I exactly: the forward's epilogues, dz = dy act'(z), and dx times act'(x_z)."""
    rng = np.random.default_rng(7)
    K = 4096 if M < 64 else 64  # from 2048 on, workgroups share the contraction of a few tokens
    lo = -8.0 if act == "gelu_tanh" else -12.5  # tanh's form falls off with the cube: below -8 nothing is left
    z = torch.from_numpy(rng.uniform(lo, 3.0, (M, K)).astype(np.float32)).to(DT)
    zr = z.double().numpy()
    z = z.cuda()
    y, g, mag = _refs(zr, act)
    note(f"tails {M} {act}")
    eye, ones = torch.eye(K, dtype=DT, device="cuda"), torch.ones(M, K, dtype=DT, device="cuda")
    kept = torch.empty_like(z)
    got = fbl.linear_fwd(z, eye, None, act, z=kept)
    assert torch.equal(kept, z)
    check("act", got, y, 2.0 ** -12 * np.abs(y) + 2.0 ** -120)
    bound = 2.0 ** -12 * mag + 2.0 ** -120
    dz = fbl.linear_bwd(ones, z, eye, z, act, need_dw=False, need_bias=False)[0]  # dz I
    check("dz", dz, g, bound)
    dx = fbl.linear_bwd(ones, z, eye, need_dw=False, need_bias=False, x_act=act, x_z=z)[0]
    check("dx", dx, g, bound)
