"""Training steps of a two-layer decoder with rotary positions, per-head norms of queries and keys, and gated feed-forward
parts, ended by clipping, through autograd: gradients and the clipped ones against the same network in float64 (torch on the
CPU), a step captured into a graph, and single tokens against the whole sequence."""
import math

import numpy as np
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import note
from paper_2607_21624_amd import autograd as ag
from test_gpu_rotary import _norm_rotary_torch
from oracle import gated_block as oracle

pytestmark = pytest.mark.gpu
B, S, H, HKV, D, L, V = 2, 72, 4, 2, 32, 2, 517
W, F = H * D, 344
EPS = 1e-5
FREQ = fbl.rotary_frequencies(D, 1000.0)


def _params(dt, seed):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s, scale=1.0, shift=0.0: (torch.randn(*s, generator=g) * scale + shift).to(dt)
    p = {"table": r(V, W, scale=0.2)}
    for i in range(L):
        p.update({f"n1w{i}": r(W, scale=0.1, shift=1.0), f"n2w{i}": r(W, scale=0.1, shift=1.0),
                  f"wqkv{i}": r(W, (H + 2 * HKV) * D, scale=W ** -0.5), f"qw{i}": r(D, scale=0.1, shift=1.0),
                  f"kw{i}": r(D, scale=0.1, shift=1.0), f"wo{i}": r(W, W, scale=W ** -0.5),
                  f"w1{i}": r(W, 2 * F, scale=W ** -0.5), f"b1{i}": r(2 * F, scale=0.1), f"w2{i}": r(F, W, scale=0.5 * F ** -0.5),
                  f"b2{i}": r(W, scale=0.1)})
    p.update(nw=r(W, scale=0.1, shift=1.0))
    return p


def _ours(p, ids, labels, turns, pos):
    x = p["table"][ids]
    for i in range(L):
        qkv = ag.linear(ag.layer_norm(x, p[f"n1w{i}"]), p[f"wqkv{i}"])
        o = ag.attention_packed(qkv, H, HKV, causal=True, turns=turns, positions=pos, q_weight=p[f"qw{i}"],
                                k_weight=p[f"kw{i}"], eps=EPS)
        x = ag.linear(o, p[f"wo{i}"], residual=x)
        h = ag.layer_norm(x, p[f"n2w{i}"])
        x = ag.gated_mlp(h, p[f"w1{i}"], p[f"b1{i}"], p[f"w2{i}"], p[f"b2{i}"], "silu", residual=x)
    return ag.linear_cross_entropy(ag.layer_norm(x, p["nw"]), p["table"].t(), labels)


def _double(p, ids, labels, pos):
    N = torch.nn.functional
    angle = torch.from_numpy(oracle.angles(pos.numpy(), FREQ))
    x = p["table"][ids]
    for i in range(L):
        q, k, v = (N.layer_norm(x, (W,), p[f"n1w{i}"]) @ p[f"wqkv{i}"]).split([H * D, HKV * D, HKV * D], dim=2)
        q = _norm_rotary_torch(q.contiguous(), H, angle, False, p[f"qw{i}"], EPS)
        k = _norm_rotary_torch(k.contiguous(), HKV, angle, False, p[f"kw{i}"], EPS)
        q, k, v = (t.reshape(B, S, -1, D).transpose(1, 2) for t in (q, k, v))
        k, v = (t.repeat_interleave(H // HKV, dim=1) for t in (k, v))
        s = (q @ k.transpose(2, 3)) / math.sqrt(D)
        s = s.masked_fill(torch.ones(S, S, dtype=torch.bool).triu(1), -math.inf)
        o = (s.softmax(3) @ v).transpose(1, 2).reshape(B, S, W)
        x = o @ p[f"wo{i}"] + x
        z = N.layer_norm(x, (W,), p[f"n2w{i}"]) @ p[f"w1{i}"] + p[f"b1{i}"]
        x = (N.silu(z[..., :F]) * z[..., F:]) @ p[f"w2{i}"] + p[f"b2{i}"] + x
    return N.cross_entropy((N.layer_norm(x, (W,), p["nw"]) @ p["table"].t()).view(-1, V), labels.view(-1))


def _batch(seed):
    rng = np.random.default_rng(seed)
    ids = torch.from_numpy(rng.integers(0, V, (B, S)))
    labels = torch.roll(ids, -1, 1)
    labels[:, -1] = -100
    labels[1, 50:] = -100  # a padded sequence
    pos = torch.arange(S).repeat(B, 1)
    pos[1] += 1000
    return ids, labels, pos


@pytest.mark.parametrize("dt,tol", [(torch.bfloat16, 2.0 ** -4), (torch.float32, 2.0 ** -14)])
def test_step(dt, tol):
    """Every gradient within `tol` of the largest of its tensor, as test_gpu_train_step.py derives it: bf16 rounds the stream
    between the 11 operators of a layer, forward and backward, some 44 half steps of 2^-8 between the table and its
    gradient, 2^-8 sqrt(44) and in the worst element 2.4 of that; fp32 2^-24 the same way and sums of up to 688 terms.  The
    clipped ones by the same, and the norm, whose errors are independent, too."""
    ids, labels, pos = _batch(3)
    p = _params(dt, 5)
    note(f"gated block step {dt}")
    mine = {k: v.cuda().requires_grad_(True) for k, v in p.items()}
    ref = {k: v.double().requires_grad_(True) for k, v in p.items()}
    a = _ours(mine, ids.cuda(), labels.cuda(), fbl.rotary_turns(FREQ), pos.cuda())
    b = _double(ref, ids, labels, pos)
    a.backward()
    b.backward()
    assert abs(a.item() - b.item()) <= tol * abs(b.item())
    off = lambda: {k: float((mine[k].grad.double().cpu() - ref[k].grad).abs().max() / ref[k].grad.abs().max()) for k in p}
    worst = off()
    assert max(worst.values()) <= tol, {k: e for k, e in worst.items() if e > tol}
    norm = math.sqrt(sum(float((t.grad ** 2).sum()) for t in ref.values()))
    got = ag.clip_grad_norm_(mine.values(), norm / 3)
    assert abs(float(got) - norm) <= tol * norm
    for t in ref.values():
        t.grad *= 1 / 3
    worst = off()
    assert max(worst.values()) <= 2 * tol, {k: e for k, e in worst.items() if e > 2 * tol}


def test_step_in_a_graph():
    """Forward, backward and clipping captured and replayed with other positions and tokens, while an eager step of other leaves
    lives; every replay is bit for bit the eager step."""
    dt = torch.bfloat16
    ids, labels, pos = (t.cuda() for t in _batch(4))
    turns = fbl.rotary_turns(FREQ)
    eager = {k: v.cuda().requires_grad_(True) for k, v in _params(dt, 6).items()}
    names = [k for k in eager if k != "table"]

    def step(p):
        loss = _ours(p, ids, labels, turns, pos)
        grads = list(torch.autograd.grad(loss, [p[k] for k in names], retain_graph=p is eager))
        return loss, fbl.clip_grad_norm(grads, 0.1), grads
    live = step(eager)
    static = {k: v.detach().clone().requires_grad_(k in names) for k, v in eager.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(static)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, norm, grads = step(static)
    for i in range(3):
        for t in grads:
            t.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, live[0]) and torch.equal(norm, live[1]) and float(norm) > 0.1
        for k, a, b in zip(names, grads, live[2]):
            assert torch.equal(a, b), k
        pos += 3
        ids.copy_(torch.roll(ids, 1, 1))
        live = step(eager)
        torch.cuda.synchronize()


def test_single_tokens_are_the_sequence_s():
    """Serving: each token's rotated query and key, and its gated part, alone at its position, are bit for bit those of the
    whole sequence (the same arithmetic in other wavefronts); the gated part within its roundings, whose contraction is
    summed in other tiles."""
    dt = torch.bfloat16
    g = torch.Generator().manual_seed(1)
    qkv = torch.randn(1, 40, (H + 2 * HKV) * D, generator=g).to(dt).cuda()
    turns, w = fbl.rotary_turns(FREQ), torch.randn(D, generator=g).to(dt).cuda()
    q, k = qkv[..., :H * D], qkv[..., H * D:(H + HKV) * D]
    how = dict(turns=turns, q_weight=w, k_weight=w, eps=EPS)
    wq, wk = fbl.qk_norm_rotary_fwd(q, k, H, HKV, **how)
    x = torch.randn(40, W, generator=g).to(dt).cuda()
    w1 = (torch.randn(W, 2 * F, generator=g) * W ** -0.5).to(dt).cuda()
    whole = fbl.gated_fwd(x, w1)
    note("single tokens of a block")
    z = x.double().cpu() @ w1.double().cpu()
    slack = (2 ** -7 * whole.double().cpu().abs()  # a rounding of each side
             + (W + 16) * 2.0 ** -22 * (x.double().cpu().abs() @ w1.double().cpu().abs()[:, :F]) * (1 + z[:, F:].abs()) + 2.0 ** -12)
    for t in (0, 1, 17, 39):
        pos = torch.tensor([[t]], device="cuda")
        a, b = fbl.qk_norm_rotary_fwd(q[:, t:t + 1], k[:, t:t + 1], H, HKV, positions=pos, **how)
        assert torch.equal(a, wq[:, t:t + 1]) and torch.equal(b, wk[:, t:t + 1])
        h = fbl.gated_fwd(x[t:t + 1], w1)
        assert torch.all((h.double().cpu() - whole[t:t + 1].double().cpu()).abs() <= slack[t:t + 1])
