"""Norms of queries and keys with their rotation, the gated feed-forward part and clipping by the global norm in float64
numpy: the textbook definitions written out (test infrastructure)."""
import math

import numpy as np

from .train import act, act_grad


# ------------------------------------------------------- per-head norm and rotation
def _pairs(D, dims, neighbours):
    """Index arrays (a, b) of the dims / 2 pairs of a head."""
    j = np.arange(dims // 2)
    return (2 * j, 2 * j + 1) if neighbours else (j, j + dims // 2)


def _scaled_turn(bits):
    """2 pi 2^bits to the nearest few integers: pi = 16 atan(1/5) - 4 atan(1/239), the series in integers."""
    def atan(n):
        term, total, k = (1 << bits + 16) // n, 0, 0
        while term:
            total += (-1) ** k * (term // (2 * k + 1))
            term //= n * n
            k += 1
        return total
    return 2 * (16 * atan(5) - 4 * atan(239)) >> 16


_BITS = 256
_TURN = _scaled_turn(_BITS)


def _reduced(n, f):
    """n f without its whole turns, within half a turn, rounded once: the product is an exact fraction, and so is what is
    left of it to 2^-256 of the turns taken away."""
    num, den = float(f).as_integer_ratio()
    turn = den * _TURN
    r = (int(n) * num << _BITS) % turn
    return (r - turn if 2 * r > turn else r) / (den << _BITS)


def angles(positions, frequencies, axes=None):
    """[B, S, dims / 2] angles from positions [B, S] or [axes, B, S]."""
    p = np.asarray(positions)
    p = p[None] if p.ndim == 2 else p
    axes = [0] * len(frequencies) if axes is None else axes
    # the whole turns go out of the product before it is rounded to float64
    return np.stack([np.vectorize(lambda n: _reduced(n, f), otypes=[np.float64])(p[a])
                     for a, f in zip(axes, frequencies)], axis=-1)


def rotate(x, angle, neighbours=False):
    """x [B, S, H, D] with its first 2 * angle.shape[-1] values turned."""
    x = np.asarray(x, dtype=np.float64)
    if angle is None:
        return x
    a, b = _pairs(x.shape[-1], 2 * angle.shape[-1], neighbours)
    c, s = np.cos(angle)[:, :, None], np.sin(angle)[:, :, None]
    y = x.copy()
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    return y


def qk_norm_rotary_fwd(x, angle=None, neighbours=False, w=None, eps=None):
    """y of x [B, S, H, D]; eps None: no norm; angle None: no rotation."""
    x = np.asarray(x, dtype=np.float64)
    if eps is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
        if w is not None:
            x = x * np.asarray(w, dtype=np.float64)
    return rotate(x, angle, neighbours)


def qk_norm_rotary_bwd(dy, x, angle=None, neighbours=False, w=None, eps=None):
    """(dx, dw)."""
    g = rotate(dy, None if angle is None else -angle, neighbours)
    if eps is None:
        return g, None
    x = np.asarray(x, dtype=np.float64)
    r = 1.0 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    xh = x * r
    dw = (g * xh).sum(axis=(0, 1, 2))
    if w is not None:
        g = g * np.asarray(w, dtype=np.float64)
    return r * (g - xh * (g * xh).mean(axis=-1, keepdims=True)), dw


# ---------------------------------------------------------------- gated feed-forward
def gated_fwd(x, w, b=None, kind="silu"):
    """(h, z): z = x w + b for w [K, 2F], gate then up;  h = act(gate) up."""
    x, w = np.asarray(x, dtype=np.float64), np.asarray(w, dtype=np.float64)
    z = x @ w
    if b is not None:
        z = z + np.asarray(b, dtype=np.float64)
    F = w.shape[1] // 2
    return act(z[:, :F], kind) * z[:, F:], z


def gated_factors(z, kind="silu"):
    """The derivatives of h by gate and by up [M, 2F]."""
    z = np.asarray(z, dtype=np.float64)
    F = z.shape[1] // 2
    return np.concatenate([z[:, F:] * act_grad(z[:, :F], kind), act(z[:, :F], kind)], axis=1)


def kept_factors(bits):
    """The values of factors as 16-bit storage holds them [M, 2F] (uint16): eight of a row share a biased exponent, whose
    bits are their bits 14, value 2q bit q and value 2q + 1 bit 4 + q; the rest is an fp16 below 1 or 1."""
    b = np.asarray(bits, dtype=np.uint16).reshape(len(bits), -1, 8)
    flags = (b >> 14 & 1).astype(np.int64)
    e = sum(flags[..., 2 * q] << q | flags[..., 2 * q + 1] << 4 + q for q in range(4))[..., None]
    half = (b & 0xBFFF).view(np.float16).astype(np.float64)
    v = np.where(e == 255, np.copysign(np.inf, half), np.ldexp(half, e - 126))
    return v.reshape(len(bits), -1)


def keep_factors(values):
    """uint16 [M, 2F] of finite fp32 values."""
    v = np.asarray(values, dtype=np.float32).reshape(len(values), -1, 8)
    e = np.abs(v).max(-1, keepdims=True).view(np.uint32).astype(np.int64) >> 23
    b = np.ldexp(v.astype(np.float64), 126 - e).astype(np.float16).view(np.uint16)
    at = np.arange(8)
    return (b | (e >> (at // 2 + at % 2 * 4) & 1) << 14).astype(np.uint16).reshape(len(values), -1)


def gated_bwd(dh, factors):
    """dz [M, 2F] from dh [M, F]."""
    dh, factors = np.asarray(dh, dtype=np.float64), np.asarray(factors, dtype=np.float64)
    return np.concatenate([dh, dh], axis=1) * factors


# ------------------------------------------------------------------------- clipping
def grad_norm(grads):
    return math.sqrt(math.fsum(float((np.asarray(g, dtype=np.float64) ** 2).sum()) for g in grads))


def clip_scale(norm, limit):
    return min(1.0, limit / (norm + 1e-6))
