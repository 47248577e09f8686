"""Linear layers and losses beside fbl_proj_tune (GPU): a workspace sized before it serves after it."""
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import note

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def untuned():
    fbl.proj_tune_reset()
    yield
    fbl.proj_tune_reset()


def _randn(*shape):
    return torch.randn(*shape, device="cuda").to(torch.bfloat16)


# The untuned tile of this weight gradient is no candidate, and beside every candidate the model would have shares of
# the contraction ahead: tuning has to leave the layout as it is.
@pytest.mark.parametrize("M,K,N", [(8000, 512, 520), (8000, 1024, 136)])
def test_a_kept_workspace_serves_after_tuning(M, K, N):
    x, w, dy = _randn(M, K), _randn(K, N) * K ** -0.5, _randn(M, N)
    note(f"tuned linear {M}x{K}x{N}")
    assert fbl.proj_auto_tile(fbl.FBL_PROJ_BWD_WEIGHT, M, K, N) not in fbl.proj_candidates(fbl.FBL_PROJ_BWD_WEIGHT, M, K, N)
    need = fbl.linear_bwd_workspace(x, w)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    z = _randn(M, N)
    before = fbl.linear_bwd(dy, x, w, z, "gelu", workspace=ws)
    plain = fbl.proj(fbl.FBL_PROJ_BWD_WEIGHT, x, dy)
    fbl.proj_tune(fbl.FBL_PROJ_BWD_WEIGHT, x, dy, torch.empty_like(w), reps=1)
    tuned = fbl.proj_tuned_tile(fbl.FBL_PROJ_BWD_WEIGHT, M, K, N)
    assert tuned >= 0 and fbl.proj_auto_tile(fbl.FBL_PROJ_BWD_WEIGHT, M, K, N) == tuned
    assert fbl.linear_bwd_workspace(x, w) == need
    after = fbl.linear_bwd(dy, x, w, z, "gelu", workspace=ws)
    assert torch.equal(before[0], after[0]) and torch.equal(before[2], after[2])
    # another tile's order of sums: each of M products of size 1 adds a rounding of at most 2^-24 of a sum below M, and
    # then half a step of the result
    assert bool(((before[1].float() - after[1].float()).abs() <= 2.0 ** -7 * before[1].float().abs() + M * 2.0 ** -10).all())
    assert plain.shape == after[1].shape


@pytest.mark.parametrize("table", [False, True])
def test_the_losses_workspace_is_of_the_shape(table):
    M, K, V = 256, 256, 16384
    x, w = _randn(M, K), _randn(V, K) if table else _randn(K, V)
    head = w.t() if table else w
    lab = torch.randint(0, V, (M,), device="cuda")
    need = fbl.linear_loss_workspace(x, head)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    note(f"tuned loss table={table}")
    dz = _randn(M, V)  # dX's product over the whole vocabulary, which is one piece
    if table:
        fbl.proj_tune(fbl.FBL_PROJ_FWD, dz, w, torch.empty_like(x), reps=1)
    else:
        fbl.proj_tune(fbl.FBL_PROJ_BWD_DATA, dz, w, torch.empty_like(x), reps=1)
    assert fbl.linear_loss_workspace(x, head) == need
    loss, lse, total = fbl.linear_ce_fwd(x, head, lab, workspace=ws)
    dx, dw = fbl.linear_ce_bwd(torch.ones((), device="cuda"), x, head, lab, lse, total, workspace=ws)
    assert bool(dx.isfinite().all()) and bool(dw.isfinite().all())
