"""A training step of a two-layer decoder made of the library's parts, through autograd:
layer norm, packed QKV projection with bias, causal GQA attention, output projection with bias and
residual, layer norm, GELU feed-forward with residual, a last layer norm and the loss on the embedding
table shared with the input -- cross entropy, or distillation from a teacher.  Gradients
against the same network in float64 (torch on the CPU)."""
import math

import numpy as np
import pytest
import torch

from ops_util import note
from paper_2607_21624_amd import autograd as ag

pytestmark = pytest.mark.gpu
B, S, H, HKV, D, L, V = 2, 72, 4, 2, 32, 2, 517
W = H * D


def _params(dt, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, scale=1.0, shift=0.0: (torch.randn(*s, generator=g) * scale + shift).to(dt)
    p = {"table": r(V, W, scale=0.2)}
    for i in range(L):
        p.update({f"n1w{i}": r(W, scale=0.1, shift=1.0), f"n1b{i}": r(W, scale=0.1), f"n2w{i}": r(W, scale=0.1, shift=1.0),
                  f"n2b{i}": r(W, scale=0.1), f"wqkv{i}": r(W, (H + 2 * HKV) * D, scale=W ** -0.5),
                  f"bqkv{i}": r((H + 2 * HKV) * D, scale=0.1), f"wo{i}": r(W, W, scale=W ** -0.5), f"bo{i}": r(W, scale=0.1),
                  f"w1{i}": r(W, 4 * W, scale=W ** -0.5), f"b1{i}": r(4 * W, scale=0.1), f"w2{i}": r(4 * W, W, scale=0.5 * W ** -0.5),
                  f"b2{i}": r(W, scale=0.1)})
    p.update(nw=r(W, scale=0.1, shift=1.0), nb=r(W, scale=0.1))
    return p


def _ours(p, ids, loss):
    x = p["table"][ids]
    for i in range(L):
        h = ag.layer_norm(x, p[f"n1w{i}"], p[f"n1b{i}"])
        qkv = ag.linear(h, p[f"wqkv{i}"], p[f"bqkv{i}"])
        o = ag.attention_packed(qkv, H, HKV, causal=True)
        x = ag.linear(o, p[f"wo{i}"], p[f"bo{i}"], residual=x)
        h = ag.layer_norm(x, p[f"n2w{i}"], p[f"n2b{i}"])
        x = ag.mlp(h, p[f"w1{i}"], p[f"b1{i}"], p[f"w2{i}"], p[f"b2{i}"], "gelu", residual=x)
    return loss(ag.layer_norm(x, p["nw"], p["nb"]), p["table"])


def _double(p, ids, loss):
    F = torch.nn.functional
    x = p["table"][ids]
    for i in range(L):
        h = F.layer_norm(x, (W,), p[f"n1w{i}"], p[f"n1b{i}"])
        q, k, v = (h @ p[f"wqkv{i}"] + p[f"bqkv{i}"]).split([H * D, HKV * D, HKV * D], dim=2)
        q, k, v = (t.view(B, S, -1, D).transpose(1, 2) for t in (q, k, v))
        k, v = (t.repeat_interleave(H // HKV, dim=1) for t in (k, v))
        s = (q @ k.transpose(2, 3)) / math.sqrt(D)
        s = s.masked_fill(torch.ones(S, S, dtype=torch.bool).triu(1), -math.inf)
        o = (s.softmax(3) @ v).transpose(1, 2).reshape(B, S, W)
        x = o @ p[f"wo{i}"] + p[f"bo{i}"] + x
        h = F.layer_norm(x, (W,), p[f"n2w{i}"], p[f"n2b{i}"])
        x = F.gelu(h @ p[f"w1{i}"] + p[f"b1{i}"]) @ p[f"w2{i}"] + p[f"b2{i}"] + x
    return loss(F.layer_norm(x, (W,), p["nw"], p["nb"]), p["table"])


@pytest.mark.parametrize("dt,tol", [(torch.bfloat16, 2.0 ** -4), (torch.float32, 2.0 ** -14)])
@pytest.mark.parametrize("kind", ["ce", "kd"])
def test_step(kind, dt, tol):
    """Every gradient within `tol` of the largest of its tensor.  bf16 rounds the stream between the 10 operators of
    a layer, forward and backward: some 40 roundings of half a step (2^-8) lie between the table and its gradient, that
    add up at random, 2^-8 sqrt(40), and in the worst element of a tensor to 2.5 of that: below 2^-4.  fp32: 2^-24
    the same way, and sums of up to 517 terms."""
    rng = np.random.default_rng(3)
    ids = torch.from_numpy(rng.integers(0, V, (B, S)))
    labels = torch.roll(ids, -1, 1)
    labels[:, -1] = -100
    labels[1, 50:] = -100  # a padded sequence
    index = torch.from_numpy(np.stack([rng.choice(V, 6, replace=False) for _ in range(B * S)]).reshape(B, S, 6))
    index[1, 50:] = -1
    logits = torch.randn(B, S, 6)
    p = _params(dt, 5)
    note(f"train step {kind} {dt}")
    mine = {k: v.cuda().requires_grad_(True) for k, v in p.items()}
    ref = {k: v.double().requires_grad_(True) for k, v in p.items()}
    if kind == "ce":
        a = _ours(mine, ids.cuda(), lambda x, t: ag.linear_cross_entropy(x, t.t(), labels.cuda()))
        b = _double(ref, ids, lambda x, t: torch.nn.functional.cross_entropy((x @ t.t()).view(-1, V), labels.view(-1)))
    else:
        a = _ours(mine, ids.cuda(), lambda x, t: ag.linear_distillation(x, t.t(), index.cuda(), logits.cuda(), 2.0))

        def kd(x, t):
            logq = torch.log_softmax(x @ t.t() / 2.0, 2)
            on = (index >= 0).all(2)
            pr = torch.softmax(logits.double() / 2.0, 2)
            each = 4 * (pr * (pr.log() - logq.gather(2, index.clamp(min=0)))).sum(2)
            return each[on].mean()
        b = _double(ref, ids, kd)
    a.backward()
    b.backward()
    assert abs(a.item() - b.item()) <= tol * abs(b.item())
    worst = {}
    for k in p:
        g, r = mine[k].grad.double().cpu(), ref[k].grad
        worst[k] = float((g - r).abs().max() / r.abs().max())
    assert max(worst.values()) <= tol, {k: e for k, e in worst.items() if e > tol}


def test_step_in_a_graph():
    """The whole step, forward and backward, captured and replayed, while an eager step of other leaves lives; the
    gradients are new tensors of the capture (torch.autograd.grad), as a captured training loop takes them."""
    dt = torch.bfloat16
    rng = np.random.default_rng(4)
    ids = torch.from_numpy(rng.integers(0, V, (B, S))).cuda()
    labels = torch.roll(ids, -1, 1)
    eager = {k: v.cuda().requires_grad_(True) for k, v in _params(dt, 6).items()}
    # the embedding's own gradient is a torch scatter; take the head's and the blocks' (a table of its own)
    run = lambda p: _ours({**p, "table": p["table"]}, ids, lambda x, t: ag.linear_cross_entropy(x, t.t(), labels))
    names = [k for k in eager if k != "table"]
    live = run(eager)  # an eager graph that stays alive
    want = [g.clone() for g in torch.autograd.grad(live, [eager[k] for k in names], retain_graph=True)]
    static = {k: v.detach().clone().requires_grad_(k in names) for k, v in eager.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.autograd.grad(run(static), [static[k] for k in names])
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        loss = run(static)
        grads = torch.autograd.grad(loss, [static[k] for k in names])
    for _ in range(3):
        for t in grads:
            t.fill_(float("nan"))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, live)
        for k, a, b in zip(names, grads, want):
            assert torch.equal(a, b), k
        assert torch.isfinite(torch.randn(1 << 16, device="cuda").sum())
