"""Results of the autograd functions changed where they stand (GPU): the values and gradients of the same step with
a new tensor in its place, bit for bit."""
import pytest
import torch

from ops_util import note
from paper_2607_21624_amd import autograd as ag

pytestmark = pytest.mark.gpu


def _leaves(seed, *shapes):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(*s, generator=g).to(torch.bfloat16).cuda().requires_grad_(True) for s in shapes]


LAYERS = {
    "linear": (ag.linear, [(64, 136)]),
    "linear_gelu": (lambda x, w, b: ag.linear(x, w, b, "gelu"), [(64, 136), (136,)]),
    "mlp": (ag.mlp, [(64, 256), (256,), (256, 64), (64,)]),
    "layer_norm": (ag.layer_norm, [(64,), (64,)]),
}


# a plain linear layer's weight gradient takes a multiple of 8 tokens, the others any number
@pytest.mark.parametrize("name,lead", [("linear", (2, 8)), ("linear", (16,))] +
                         [(n, lead) for n in LAYERS if n != "linear" for lead in ((3, 5), (15,), ())])
def test_layers(name, lead):
    f, shapes = LAYERS[name]
    leaves = _leaves(1, (*lead, 64), *shapes)
    note(f"in place {name} {lead}")
    y = f(*leaves)
    assert y.shape[:-1] == lead and y.is_contiguous()
    want = torch.autograd.grad(y * 2, leaves, torch.ones_like(y))
    z = f(*leaves)
    z *= 2
    assert torch.equal(z, y * 2)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(z, leaves, torch.ones_like(z)), want))


@pytest.mark.parametrize("reduction", ["mean", "sum", "none"])
@pytest.mark.parametrize("kind", ["ce", "kd"])
def test_losses(kind, reduction):
    x, table = _leaves(2, (3, 7, 64), (200, 64))
    ids = torch.randint(0, 200, (3, 7, 4), generator=torch.Generator().manual_seed(3)).cuda()
    labels = ids[..., 0].contiguous()
    logits = torch.randn(3, 7, 4, generator=torch.Generator().manual_seed(4)).cuda()
    note(f"in place loss {kind} {reduction}")

    def run():
        if kind == "ce":
            return ag.linear_cross_entropy(x, table.t(), labels, reduction=reduction)
        return ag.linear_distillation(x, table.t(), ids, logits, 2.0, reduction)
    loss = run()
    assert loss.shape == ((3, 7) if reduction == "none" else ())
    want = torch.autograd.grad(loss / 4, [x, table], torch.ones_like(loss))
    again = run()
    again /= 4
    assert torch.equal(again, loss / 4)
    got = torch.autograd.grad(again, [x, table], torch.ones_like(again))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
