"""Linear layers whose operands end inside a 16-byte chunk, against the float64 oracle with test_gpu_linear.py's
bounds (GPU)."""
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import padded
from test_gpu_linear import _case, _check_bwd, _check_fwd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["relu", "gelu"])
@pytest.mark.parametrize("M,K,N", [(1, 64, 4), (77, 264, 260), (301, 2056, 268), (8200, 128, 68), (9001, 72, 132)])
def test_weight_gradient_of_a_width_that_ends_inside_a_chunk(M, K, N, act):
    """N % 8 == 4, dw and dbias alone, behind an activation: dz is an operand of its own in the workspace; its
    contraction shared (the narrow ones of many tokens) and not, operands and dw between guards."""
    dt = torch.bfloat16
    (x, w, b, _, dy), ref = _case(M, K, N, dt, act, True, False)
    row = lambda t: padded(t, 4)[0]  # rows of N + 4
    z = row(torch.zeros(M, N, dtype=dt, device="cuda"))
    y = fbl.linear_fwd(x, row(w), b, act, out=row(torch.zeros(M, N, dtype=dt, device="cuda")), z=z)
    zr, zb = _check_fwd(y, z, ref, act, dt)
    view, buf = padded(torch.zeros(K, N, dtype=dt, device="cuda"), 4, 7.0)
    ws = torch.full((fbl.linear_bwd_workspace(x, w),), 0xff, dtype=torch.uint8, device="cuda")
    _, dw, db = fbl.linear_bwd(row(dy), x, row(w), z, act, dw=view, need_dx=False, workspace=ws)
    _check_bwd(None, dw, db, ref, zr, zb, act, dt)
    assert bool((buf[:, N:] == 7.0).all()) and bool((buf[-1] == 7.0).all())
