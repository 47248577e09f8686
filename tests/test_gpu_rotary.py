"""Norms of queries and keys for each head with their rotation, forward and backward, against the float64 oracle (GPU).

Bounds, element by element, in half steps of fp32, u = 2^-24.  A turned value is a c - b s of its pair: off by
the cosine's and sine's error times |a| + |b|, and 3 roundings.  fp32: the angle within a quarter turn is at most pi / 4, kept
to 2^-32 turns, rounded to fp32 and scaled (2.4 u); the polynomials are good to 2e-9 and their last steps round twice:
below 6 u; with the products 9 u.  bf16: the hardware's cosine and sine, taken to be good to 2^-17, a
sixtieth of the storage's half step.  The norm: a sum of squares of at most 16 terms in a lane and 4 steps across lanes, 20 u of
itself, half of that through the square root, division, root and products 5 u: r x w is good to 16 u.  Its backward sums g x r the
same way (20 u of the sum of magnitudes), and rounds 6 times more.  The weights' gradients add tokens * heads terms, in a
lane at most `steps` after one another, then 5 steps across lanes, 3 across wavefronts, workgroups / 32 and 32."""
import numpy as np
import pytest
import torch

import paper_2607_21624_amd as fbl
from ops_util import DTYPES, check, note, rounded
from oracle import gated_block as oracle

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def trig(dt):
    return 2.0 ** -17 if dt == torch.bfloat16 else 9 * U


def _pair_sum(x, dims, neighbours):
    """|a| + |b| of each value's pair, its own magnitude where it does not turn."""
    m = np.abs(x)
    y = m.copy()
    if dims:
        a, b = oracle._pairs(x.shape[-1], dims, neighbours)
        y[..., a] = y[..., b] = m[..., a] + m[..., b]
    return y


def _heads(x, H):
    return x.reshape(*x.shape[:2], H, -1)


def _make(B, S, Hq, Hkv, d, dt, rng, scale=1.5):
    qkv, r = rounded(rng, (B, S, (Hq + 2 * Hkv) * d), dt, scale)
    return qkv, r, (slice(0, Hq * d), slice(Hq * d, (Hq + Hkv) * d))


def _run(B, S, Hq, Hkv, d, dt, dims, neighbours=False, norm=True, weights=True, positions=None, axes=None, freq=None,
         separate=False, eps=1e-6, seed=0):
    rng = np.random.default_rng(seed + 7 * S + d)
    qkv, r, cols = _make(B, S, Hq, Hkv, d, dt, rng)
    g, gr = rounded(rng, (B, S, (Hq + Hkv) * d), dt)
    wq, wqr = rounded(rng, (d,), dt, 0.2, 1.0) if norm and weights else (None, None)
    wk, wkr = rounded(rng, (d,), dt, 0.2, 1.0) if norm and weights else (None, None)
    freq = fbl.rotary_frequencies(dims) if freq is None else freq
    turns = fbl.rotary_turns(freq) if dims else None
    note(f"qk_norm_rotary B={B} S={S} Hq={Hq} Hkv={Hkv} d={d} {dt} dims={dims} neighbours={neighbours} norm={norm}")
    pos = np.broadcast_to(np.arange(S), (B, S)) if positions is None else positions
    how = dict(turns=turns, positions=None if positions is None else torch.from_numpy(np.array(positions)).cuda(), axes=axes,
               neighbours=neighbours, q_weight=wq, k_weight=wk, eps=eps if norm else None)
    q, k = qkv[..., cols[0]], qkv[..., cols[1]]
    gq, gk = g[..., :Hq * d], g[..., Hq * d:]
    if separate:
        q, k, gq, gk = (t.contiguous() for t in (q, k, gq, gk))
    yq, yk = fbl.qk_norm_rotary_fwd(q, k, Hq, Hkv, **how)
    dqkv = torch.full_like(qkv, 9.0)
    dq, dk, dqw, dkw = fbl.qk_norm_rotary_bwd(gq, gk, q, k, Hq, Hkv, dq=dqkv[..., cols[0]], dk=dqkv[..., cols[1]], **how)
    torch.cuda.synchronize()
    assert torch.all(dqkv[..., (Hq + Hkv) * d:] == 9.0)
    angle = oracle.angles(np.array(pos), freq, axes) if dims else None
    t = trig(dt) if dims else 0.0
    for name, y, dx, dw, x, dy, w, H in (("q", yq, dq, dqw, r[..., cols[0]], gr[..., :Hq * d], wqr, Hq),
                                         ("k", yk, dk, dkw, r[..., cols[1]], gr[..., Hq * d:], wkr, Hkv)):
        x, dy = _heads(x, H), _heads(dy, H)
        e = eps if norm else None
        h = oracle.qk_norm_rotary_fwd(x, None, w=w, eps=e)
        ref = oracle.qk_norm_rotary_fwd(x, angle, neighbours, w, e)
        check(f"{name}'", y, ref.reshape(B, S, -1), ((t + (16 * U if norm else 0)) * _pair_sum(h, dims, neighbours)).reshape(B, S, -1))
        dxr, dwr = oracle.qk_norm_rotary_bwd(dy, x, angle, neighbours, w, e)
        G = _pair_sum(dy, dims, neighbours)  # of the gradient turned back
        if not norm:
            assert dw is None
            check(f"d{name}", dx, dxr.reshape(B, S, -1), (t * G).reshape(B, S, -1))
            continue
        rstd = 1.0 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
        xh, gw = np.abs(x * rstd), G * (1.0 if w is None else np.abs(w))
        terms = gw + xh * (gw * xh).mean(-1, keepdims=True)
        check(f"d{name}", dx, dxr.reshape(B, S, -1), ((t + 60 * U) * rstd * terms).reshape(B, S, -1))
        if w is None:
            assert dw is None
        else:
            chain = B * S / 1024 * (H * d / 512 + 1) + H + 64 + 32
            check(f"d{name}_weight", dw, dwr, (t + (20 + chain) * U) * (G * xh).sum((0, 1, 2)))
    return qkv, how, (yq, yk), (dq, dk, dqw, dkw)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("d", [32, 64, 128])
@pytest.mark.parametrize("neighbours", [False, True])
def test_heads_and_pairs(dt, d, neighbours):
    dt = DTYPES[dt]
    for Hq, Hkv, S in ((4, 2, 37), (1, 1, 1), (5, 5, 3), (12, 4, 130)):
        _run(2, S, Hq, Hkv, d, dt, d, neighbours)
    _run(1, 19, 40, 8, d, dt, 16, neighbours)           # a part of a head turns
    _run(3, 5, 3, 1, d, dt, d // 2, neighbours, norm=False)
    _run(1, 9, 2, 2, d, dt, 0, neighbours)              # the norm alone
    _run(2, 6, 6, 2, d, dt, d, neighbours, weights=False, separate=True)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_far_and_negative_positions(dt):
    rng = np.random.default_rng(5)
    far = rng.integers(0, 1 << 40, (4, 3))
    far[0] = [0, 1, -1]
    far[1] = [(1 << 31) - 1, 1 << 31, -(1 << 31)]
    far[2] = [1 << 32, (1 << 32) + 1, 123456789012]
    # whole 64ths of a turn a position, so that the oracle's angles are exact
    steps = (1, 5, 7, 13, 17, 23, 29, 63)
    turns = torch.tensor([(k << 58) - (1 << 64) * (k >= 32) for k in steps], device="cuda")
    dt = DTYPES[dt]
    q, qr = rounded(rng, (4, 3, 2 * 32), dt)
    note(f"far positions {dt}")
    y, none = fbl.qk_norm_rotary_fwd(q, None, 2, 0, turns=turns, positions=torch.from_numpy(far).cuda())
    assert none is None
    angle = np.stack([(far % 64) * k % 64 * (2 * np.pi / 64) for k in steps], axis=-1)
    x = _heads(qr, 2)
    check("y", y, oracle.rotate(x, angle).reshape(4, 3, -1), (trig(dt) * _pair_sum(x, 16, False)).reshape(4, 3, -1))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("base", [1e4, 5e5])
def test_ordinary_frequencies_at_far_positions(dt, base):
    """Up to 2^31 positions from 0.  The kept frequency is off by the quotient's roundings, 2^-63 of at most 1 / 2 pi of a turn,
    and its own, 2^-65 turns: 2^31 positions make that 0.82 2^-33 turns, 6e-10 or 0.0101 u."""
    rng = np.random.default_rng(15)
    dt = DTYPES[dt]
    far = rng.integers(-(1 << 31), 1 << 31, (3, 40))
    far[0, :6] = [0, (1 << 31) - 1, -(1 << 31), 10 ** 9 + 7, 1 << 30, -(1 << 20) - 1]
    freq = fbl.rotary_frequencies(64, base)
    q, qr = rounded(rng, (3, 40, 2 * 64), dt)
    note(f"ordinary frequencies at far positions {dt}")
    y, _ = fbl.qk_norm_rotary_fwd(q, None, 2, 0, turns=fbl.rotary_turns(freq), positions=torch.from_numpy(far).cuda())
    x = _heads(qr, 2)
    check("y", y, oracle.rotate(x, oracle.angles(far, freq)).reshape(3, 40, -1), ((trig(dt) + 0.0101 * U) * _pair_sum(x, 64, False)).reshape(3, 40, -1))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_single_tokens_at_their_positions(dt):
    rng = np.random.default_rng(6)
    for B in (1, 7, 200):
        _run(B, 1, 32, 8, 64, DTYPES[dt], 64, norm=False, positions=rng.integers(0, 1 << 20, (B, 1)), freq=fbl.rotary_frequencies(64, 5e5))
        _run(B, 1, 4, 4, 128, DTYPES[dt], 128, positions=rng.integers(0, 1 << 17, (B, 1)))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_axes(dt):
    rng = np.random.default_rng(8)
    pos = rng.integers(0, 300, (3, 2, 21))
    _run(2, 21, 4, 2, 64, DTYPES[dt], 64, positions=pos, axes=[0] * 8 + [1] * 12 + [2] * 12)
    _run(2, 21, 3, 3, 128, DTYPES[dt], 32, True, positions=pos, axes=[i % 3 for i in range(16)])
    pos = rng.integers(0, 300, (4, 2, 21))
    _run(2, 21, 2, 1, 128, DTYPES[dt], 128, positions=pos, axes=[(i * 7) % 4 for i in range(64)])


def test_positions_given_as_views():
    rng = np.random.default_rng(9)
    q, _ = rounded(rng, (3, 8, 2 * 64), torch.bfloat16)
    k, _ = rounded(rng, (3, 8, 1 * 64), torch.bfloat16)
    turns = fbl.rotary_turns(fbl.rotary_frequencies(64))
    base = torch.arange(8, device="cuda")
    run = lambda p, **kw: fbl.qk_norm_rotary_fwd(q, k, 2, 1, turns=turns, positions=p, **kw)
    want = run(None)
    wide = torch.zeros(8, 3, 5, dtype=torch.int64, device="cuda")
    wide[..., 2] = base[:, None]
    three = base.expand(3, 3, 8)
    for p, kw in ((base, {}), (base.expand(3, 8), {}), (wide[..., 2].t(), {}), (base.expand(1, 3, 8), {}),
                  (three, dict(axes=[i % 3 for i in range(32)]))):
        got = run(p, **kw)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("norm", [False, True])
def test_in_place(dt, norm):
    qkv, how, (yq, yk), (dq, dk, dqw, dkw) = _run(2, 33, 6, 2, 64, DTYPES[dt], 64, norm=norm)
    own = qkv.clone()
    q, k, v = own[..., :384], own[..., 384:512], own[..., 512:]
    fbl.qk_norm_rotary_fwd(q, k, 6, 2, q_out=q, k_out=k, **how)
    assert torch.equal(q, yq) and torch.equal(k, yk) and torch.equal(v, qkv[..., 512:])
    # the gradient where attention leaves it
    rng = np.random.default_rng(7 * 33 + 64)
    _make(2, 33, 6, 2, 64, DTYPES[dt], rng)
    g, _ = rounded(rng, (2, 33, 8 * 64), DTYPES[dt])
    packed = torch.full_like(qkv, 3.0)
    packed[..., :512] = g
    gq, gk = packed[..., :384], packed[..., 384:512]
    out = fbl.qk_norm_rotary_bwd(gq, gk, qkv[..., :384], qkv[..., 384:512], 6, 2, dq=gq, dk=gk, **how)
    assert torch.equal(gq, dq) and torch.equal(gk, dk) and torch.all(packed[..., 512:] == 3.0)
    if norm:
        assert torch.equal(out[2], dqw) and torch.equal(out[3], dkw)


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("S,Hq,Hkv,d", [(5, 3, 2, 64), (7, 1, 1, 32), (1, 5, 0, 128), (3, 11, 3, 32), (1, 1, 1, 64)])
def test_in_place_where_lanes_have_no_head_or_token(dt, S, Hq, Hkv, d):
    """Lanes behind the last head and token repeat its work: in place too, with nothing written behind it, and nothing added
    twice."""
    dtype = DTYPES[dt]
    rng = np.random.default_rng(31 + S)
    W = (Hq + Hkv) * d
    x, xr = rounded(rng, (1, S, W), dtype)
    g, gr = rounded(rng, (1, S, W), dtype)
    w, wr = rounded(rng, (d,), dtype, 0.2, 1.0)
    how = dict(turns=fbl.rotary_turns(fbl.rotary_frequencies(d)), q_weight=w, k_weight=w if Hkv else None, eps=1e-6)
    split = lambda t: (t[..., :Hq * d], t[..., Hq * d:W] if Hkv else None)
    note(f"in place, S={S} heads {Hq} + {Hkv} of {d} {dt}")
    want = fbl.qk_norm_rotary_fwd(*split(x), Hq, Hkv, **how)
    grads = fbl.qk_norm_rotary_bwd(*split(g), *split(x), Hq, Hkv, **how)
    _, dw = oracle.qk_norm_rotary_bwd(_heads(gr[..., :Hq * d], Hq), _heads(xr[..., :Hq * d], Hq),
                                      oracle.angles(np.arange(S)[None], fbl.rotary_frequencies(d), None), False, wr, 1e-6)
    xh = _heads(xr[..., :Hq * d], Hq)
    xh = np.abs(xh / np.sqrt((xh * xh).mean(-1, keepdims=True) + 1e-6))
    check("dw", grads[2], dw, (trig(dtype) + 160 * U) * (_pair_sum(_heads(gr[..., :Hq * d], Hq), d, False) * xh).sum((0, 1, 2)))
    for back in (False, True):
        buf = torch.full((1, S + 2, W + 16), 7.0, dtype=dtype, device="cuda")
        own = buf[:, :S, :W]
        own.copy_(g if back else x)
        q, k = split(own)
        if back:
            got = fbl.qk_norm_rotary_bwd(q, k, *split(x), Hq, Hkv, dq=q, dk=k, **how)
        else:
            got = fbl.qk_norm_rotary_fwd(q, k, Hq, Hkv, q_out=q, k_out=k, **how)
        for a, b in zip(got, grads if back else want):
            assert (a is None and b is None) or torch.equal(a, b)
        assert torch.all(buf[:, S:] == 7.0) and torch.all(buf[..., W:] == 7.0)


def test_repeatable_and_need_not():
    rng = np.random.default_rng(3)
    q, _ = rounded(rng, (2, 700, 8 * 64), torch.bfloat16)
    g, _ = rounded(rng, (2, 700, 8 * 64), torch.bfloat16)
    w, _ = rounded(rng, (64,), torch.bfloat16, 0.2, 1.0)
    note("qk_norm_rotary repeatable")
    f = lambda **kw: fbl.qk_norm_rotary_bwd(g, None, q, None, 8, 0, q_weight=w, eps=1e-6, **kw)
    a, b = f(), f()
    assert torch.equal(a[0], b[0]) and torch.equal(a[2], b[2]) and a[1] is None and a[3] is None
    c = f(need_weights=False)
    assert torch.equal(a[0], c[0]) and c[2] is None
    ws = torch.full((fbl.qk_norm_rotary_bwd_workspace(q, None, 8, 0),), 255, dtype=torch.uint8, device="cuda")
    assert torch.equal(f(workspace=ws)[2], a[2])


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_infinite_values_stay_in_their_head(dt):
    dt = DTYPES[dt]
    rng = np.random.default_rng(4)
    q, _ = rounded(rng, (1, 6, 4 * 64), dt)
    turns = fbl.rotary_turns(fbl.rotary_frequencies(32))
    clean = fbl.qk_norm_rotary_fwd(q, None, 4, 0, turns=turns, eps=1e-6)[0]
    bad = q.clone()
    bad[0, 2, 64 + 40] = float("inf")
    bad[0, 4, 128 + 3] = float("nan")
    note(f"infinite values {dt}")
    got = fbl.qk_norm_rotary_fwd(bad, None, 4, 0, turns=turns, eps=1e-6)[0]
    keep = torch.ones_like(q, dtype=torch.bool)
    keep[0, 2, 64:128] = keep[0, 4, 128:192] = False
    assert torch.equal(got[keep], clean[keep])
    # without the norm a value that does not turn stays alone, and one that does reaches its pair
    got = fbl.qk_norm_rotary_fwd(bad, None, 4, 0, turns=turns)[0]
    clean = fbl.qk_norm_rotary_fwd(q, None, 4, 0, turns=turns)[0]
    keep = torch.ones_like(q, dtype=torch.bool)
    keep[0, 2, 64 + 40] = False
    keep[0, 4, 128 + 3] = keep[0, 4, 128 + 19] = False
    assert torch.equal(got[keep], clean[keep]) and torch.isinf(got[0, 2, 104])
    # a head of zeros with eps 0 is 0 / 0, and reaches nothing else, the weights' gradients excepted
    zero = q.clone()
    zero[0, 1, :64] = 0
    got = fbl.qk_norm_rotary_fwd(zero, None, 4, 0, eps=0.0)[0]
    assert torch.isnan(got[0, 1, :64]).all() and not torch.isnan(got[0, 1, 64:]).any()


def test_dead_lanes_leave_the_sums():
    # 3 heads of 8 lanes: five lane groups of the wavefront have no head, and eps is 0
    rng = np.random.default_rng(11)
    q, qr = rounded(rng, (1, 5, 3 * 128), torch.bfloat16)
    g, gr = rounded(rng, (1, 5, 3 * 128), torch.bfloat16)
    w, wr = rounded(rng, (128,), torch.bfloat16, 0.2, 1.0)
    note("dead lanes")
    _, _, dw, _ = fbl.qk_norm_rotary_bwd(g, None, q, None, 3, 0, q_weight=w, eps=0.0)
    _, ref = oracle.qk_norm_rotary_bwd(_heads(gr, 3), _heads(qr, 3), w=wr, eps=0.0)
    xh = np.abs(_heads(qr, 3)) / np.sqrt((_heads(qr, 3) ** 2).mean(-1, keepdims=True))
    check("dw", dw, ref, 120 * U * (np.abs(_heads(gr, 3)) * xh).sum((0, 1, 2)))


@pytest.mark.parametrize("dt", ["bf16", "f32"])
@pytest.mark.parametrize("S,Hq,Hkv,d", [(5, 3, 0, 128), (3, 1, 1, 32), (7, 40, 8, 64), (4, 2, 3, 64), (1, 1, 1, 128)])
def test_an_infinite_gradient_stays_in_its_column_of_the_weights(dt, S, Hq, Hkv, d):
    """An infinite value of dy that does not turn, times a finite r x: the weight's gradient is infinite there, of r x's sign, and
    what it was in all other columns, also where lanes without a head or token repeat the head."""
    dtype = DTYPES[dt]
    rng = np.random.default_rng(41 + S)
    W, dims = (Hq + Hkv) * d, 16
    x, xr = rounded(rng, (1, S, W), dtype)
    g, _ = rounded(rng, (1, S, W), dtype)
    w, _ = rounded(rng, (d,), dtype, 0.2, 1.0)
    how = dict(turns=fbl.rotary_turns(fbl.rotary_frequencies(dims)), q_weight=w, k_weight=w if Hkv else None, eps=1e-6)
    split = lambda t: (t[..., :Hq * d], t[..., Hq * d:] if Hkv else None)
    note(f"infinite gradient, S={S} heads {Hq} + {Hkv} of {d} {dt}")
    clean = fbl.qk_norm_rotary_bwd(*split(g), *split(x), Hq, Hkv, **how)
    col = dims + 5
    for head, i in ((Hq - 1, 2), (Hq + Hkv - 1, 3 if Hkv else 2)):  # the last ones, which are repeated
        for value in (float("inf"), float("-inf")):
            bad = g.clone()
            bad[0, S - 1, head * d + col] = value
            got = fbl.qk_norm_rotary_bwd(*split(bad), *split(x), Hq, Hkv, **how)
            want = clean[i].float().clone()
            want[col] = value * np.sign(xr[0, S - 1, head * d + col])
            assert torch.equal(got[i].float(), want)
            other = 5 - i
            assert clean[other] is None or torch.equal(got[other], clean[other])


def test_offsets_past_32_bits():
    # a batch is 2^32 bytes and more from the next one, a token 2^31
    rng = np.random.default_rng(13)
    q, _ = rounded(rng, (2, 2, 4 * 64), torch.bfloat16)
    k, _ = rounded(rng, (2, 2, 2 * 64), torch.bfloat16)
    w, _ = rounded(rng, (64,), torch.bfloat16, 0.2, 1.0)
    how = dict(turns=fbl.rotary_turns(fbl.rotary_frequencies(64)), q_weight=w, k_weight=w, eps=1e-6)
    ss, sb = 1 << 30, 1 << 31
    buf = torch.empty(sb + ss + 1024, dtype=torch.bfloat16, device="cuda")
    far = lambda t, col: buf.as_strided(t.shape, (sb, ss, 1), col).copy_(t)
    fq, fk = far(q, 0), far(k, 256)
    gq, gk = far(k.repeat(1, 1, 2), 384), far(q[..., 128:], 640)
    note("qk_norm_rotary past 32 bits")
    want = fbl.qk_norm_rotary_bwd(gq.contiguous(), gk.contiguous(), q, k, 4, 2, **how)
    got = fbl.qk_norm_rotary_bwd(gq, gk, fq, fk, 4, 2, dq=gq, dk=gk, **how)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    want = fbl.qk_norm_rotary_fwd(q, k, 4, 2, **how)
    got = fbl.qk_norm_rotary_fwd(fq, fk, 4, 2, q_out=fq, k_out=fk, **how)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_on_another_stream():
    rng = np.random.default_rng(14)
    q, _ = rounded(rng, (2, 65, 4 * 64), torch.bfloat16)
    k, _ = rounded(rng, (2, 65, 64), torch.bfloat16)
    w, _ = rounded(rng, (64,), torch.bfloat16, 0.2, 1.0)
    how = dict(turns=fbl.rotary_turns(fbl.rotary_frequencies(64)), q_weight=w, k_weight=w, eps=1e-6)
    run = lambda **kw: (*fbl.qk_norm_rotary_fwd(q, k, 4, 1, **how, **kw), *fbl.qk_norm_rotary_bwd(q, k, q, k, 4, 1, **how, **kw))
    want = run()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    note("qk_norm_rotary on another stream")
    given = run(stream=side)
    with torch.cuda.stream(side):
        current = run()
    torch.cuda.synchronize()
    for got in (given, current):
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------------ autograd
def _norm_rotary_torch(x, H, angle, neighbours, w, eps):
    """The same in torch, float64 on the CPU."""
    B, S, _ = x.shape
    h = x.view(B, S, H, -1)
    d = h.shape[-1]
    if eps is not None:
        h = h / torch.sqrt((h * h).mean(-1, keepdim=True) + eps) * w
    c, s = torch.cos(angle)[:, :, None], torch.sin(angle)[:, :, None]
    n = 2 * angle.shape[-1]
    a, b = (h[..., 0:n:2], h[..., 1:n:2]) if neighbours else (h[..., :n // 2], h[..., n // 2:n])
    u, v = a * c - b * s, b * c + a * s
    t = torch.stack([u, v], -1).flatten(-2) if neighbours else torch.cat([u, v], -1)
    return torch.cat([t, h[..., n:]], -1).reshape(B, S, H * d)


@pytest.mark.parametrize("dt,neighbours", [("bf16", False), ("f32", True)])
def test_autograd_attention_packed(dt, neighbours):
    from paper_2607_21624_amd import autograd as ag
    dtype = DTYPES[dt]
    B, S, Hq, Hkv, d = 2, 70, 4, 2, 64
    rng = np.random.default_rng(12)
    qkv, qkvr, _ = _make(B, S, Hq, Hkv, d, dtype, rng, 1.0)
    wq, wqr = rounded(rng, (d,), dtype, 0.2, 1.0)
    wk, wkr = rounded(rng, (d,), dtype, 0.2, 1.0)
    do, dor = rounded(rng, (B, S, Hq * d), dtype)
    freq = fbl.rotary_frequencies(d)
    how = dict(turns=fbl.rotary_turns(freq), neighbours=neighbours, q_weight=wq, k_weight=wk, eps=1e-6)
    note(f"attention_packed with rotary {dt}")
    leaves = [t.requires_grad_(True) for t in (qkv, wq, wk)]
    o = ag.attention_packed(qkv, Hq, Hkv, causal=True, **how)
    got = torch.autograd.grad(o, leaves, do)
    # bit for bit the explicit calls
    q, k, v = (t.detach() for t in (qkv[..., :Hq * d], qkv[..., Hq * d:(Hq + Hkv) * d], qkv[..., (Hq + Hkv) * d:]))
    with torch.no_grad():
        yq, yk = fbl.qk_norm_rotary_fwd(q, k, Hq, Hkv, **how)
        o2, lse = fbl.attn_fwd(yq, yk, v, Hq, Hkv, causal=True)
        dq, dk, dv = fbl.attn_bwd(yq, yk, v, o2, do, lse, Hq, Hkv, causal=True)
        dq, dk, dqw, dkw = fbl.qk_norm_rotary_bwd(dq, dk, q, k, Hq, Hkv, **how)
    assert torch.equal(o, o2) and torch.equal(got[0], torch.cat([dq, dk, dv], -1))
    assert torch.equal(got[1], dqw) and torch.equal(got[2], dkw)
    # and through the function of its own
    yq, yk = ag.qk_norm_rotary(qkv[..., :Hq * d], qkv[..., Hq * d:(Hq + Hkv) * d], Hq, Hkv, **how)
    o3 = ag.attention(yq, yk, qkv[..., (Hq + Hkv) * d:], Hq, Hkv, causal=True)
    assert torch.equal(o3, o2)
    got3 = torch.autograd.grad(o3, leaves, do)
    assert all(torch.equal(a, b) for a, b in zip(got, got3))
    # float64: the tolerance of attention's own tests, relative to the largest value
    x64 = torch.from_numpy(qkvr).requires_grad_(True)
    w64 = [torch.from_numpy(w).requires_grad_(True) for w in (wqr, wkr)]
    angle = torch.from_numpy(oracle.angles(np.broadcast_to(np.arange(S), (B, S)), freq))
    q64 = _norm_rotary_torch(x64[..., :Hq * d], Hq, angle, neighbours, w64[0], 1e-6).view(B, S, Hq, d).transpose(1, 2)
    k64 = _norm_rotary_torch(x64[..., Hq * d:(Hq + Hkv) * d], Hkv, angle, neighbours, w64[1], 1e-6).view(B, S, Hkv, d).transpose(1, 2)
    v64 = x64[..., (Hq + Hkv) * d:].view(B, S, Hkv, d).transpose(1, 2)
    k64, v64 = k64.repeat_interleave(Hq // Hkv, 1), v64.repeat_interleave(Hq // Hkv, 1)
    p = (q64 @ k64.transpose(-1, -2) / d ** 0.5).masked_fill(~torch.tril(torch.ones(S, S, dtype=torch.bool)), -torch.inf).softmax(-1)
    o64 = (p @ v64).transpose(1, 2).reshape(B, S, Hq * d)
    ref = torch.autograd.grad(o64, [x64, *w64], torch.from_numpy(dor))
    tol = 2e-2 if dt == "bf16" else 1e-4
    for a, b in zip((o, *got), (o64, *ref)):
        b = b.detach()
        assert float((a.detach().double().cpu() - b).abs().max()) <= tol * float(b.abs().max())


def test_autograd_keys_alone_unused_and_second_order():
    from paper_2607_21624_amd import autograd as ag
    rng = np.random.default_rng(13)
    q = rounded(rng, (2, 9, 128), torch.float32)[0].requires_grad_(True)
    k = rounded(rng, (2, 9, 64), torch.float32)[0].requires_grad_(True)
    turns = fbl.rotary_turns(fbl.rotary_frequencies(64))
    note("qk_norm_rotary autograd corners")
    yq, yk = ag.qk_norm_rotary(q, k, 2, 1, turns=turns)
    dq, dk = torch.autograd.grad(yk, (q, k), torch.ones_like(yk))  # nothing depends on q'
    assert torch.all(dq == 0) and torch.equal(dk, fbl.qk_norm_rotary_bwd(torch.ones_like(yk), None, None, None, 1, 0, turns=turns)[0])
    y, none = ag.qk_norm_rotary(q, None, 2, 0, turns=turns, eps=1e-6)
    assert none is None
    (g,) = torch.autograd.grad(y, q, torch.ones_like(y), create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()
    y, _ = ag.qk_norm_rotary(q, None, 2, 0, turns=turns)
    y *= 2  # its backward reads no result
    assert torch.isfinite(torch.autograd.grad(y, q, torch.ones_like(y))[0]).all()


def test_graph_replays():
    rng = np.random.default_rng(14)
    q, _ = rounded(rng, (2, 65, 4 * 64), torch.bfloat16)
    g, _ = rounded(rng, (2, 65, 4 * 64), torch.bfloat16)
    w, _ = rounded(rng, (64,), torch.bfloat16, 0.2, 1.0)
    pos = torch.arange(65, device="cuda").repeat(2, 1)
    how = dict(turns=fbl.rotary_turns(fbl.rotary_frequencies(64)), positions=pos, q_weight=w, eps=1e-6)
    y, dx, dw = torch.empty_like(q), torch.empty_like(q), torch.empty_like(w)
    ws = torch.empty(fbl.qk_norm_rotary_bwd_workspace(q, None, 4, 0), dtype=torch.uint8, device="cuda")
    note("qk_norm_rotary graph")

    def step():
        fbl.qk_norm_rotary_fwd(q, None, 4, 0, q_out=y, **how)
        fbl.qk_norm_rotary_bwd(g, None, q, None, 4, 0, dq=dx, dq_weight=dw, workspace=ws, **how)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        q.copy_(rounded(rng, tuple(q.shape), torch.bfloat16)[0])
        pos += 1000  # read anew by every replay
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw)))
