"""Layer norm, linear layers with an epilogue and the losses of a linear head in
float64 numpy: the textbook definitions written out (test infrastructure)."""
import math

import numpy as np


def _f64(*a):
    return tuple(None if x is None else np.asarray(x, dtype=np.float64) for x in a)


# ---------------------------------------------------------------- layer norm
def layer_norm_fwd(x, w=None, b=None, eps=1e-5):
    """(y, mean, rstd) over the last axis of x [M, N]."""
    x, w, b = _f64(x, w, b)
    mean = x.mean(axis=1)
    rstd = 1.0 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    if w is not None:
        y = y * w
    if b is not None:
        y = y + b
    return y, mean, rstd


def layer_norm_bwd(dy, x, w=None, eps=1e-5):
    """(dx, dw, db)."""
    dy, x, w = _f64(dy, x, w)
    xh, _, rstd = layer_norm_fwd(x, eps=eps)
    g = dy if w is None else dy * w
    dx = rstd[:, None] * (g - g.mean(axis=1, keepdims=True) - xh * (g * xh).mean(axis=1, keepdims=True))
    return dx, (dy * xh).sum(axis=0), dy.sum(axis=0)


# ------------------------------------------------------------ linear + epilogue
def _erf(z):
    return np.vectorize(math.erf, otypes=[np.float64])(z)


def act(z, kind):
    (z,) = _f64(z)
    if kind == "none":
        return z
    if kind == "relu":
        return np.where(z > 0, z, 0.0)
    if kind == "gelu":
        return 0.5 * z * (1.0 + _erf(z / math.sqrt(2.0)))
    if kind == "gelu_tanh":
        return 0.5 * z * (1.0 + np.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    if kind == "silu":
        return z / (1.0 + np.exp(-z))
    raise ValueError(kind)


def act_grad(z, kind):
    (z,) = _f64(z)
    if kind == "none":
        return np.ones_like(z)
    if kind == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if kind == "gelu":
        return 0.5 * (1.0 + _erf(z / math.sqrt(2.0))) + z * np.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if kind == "gelu_tanh":
        c, a = math.sqrt(2.0 / math.pi), 0.044715
        t = np.tanh(c * (z + a * z ** 3))
        return 0.5 * (1.0 + t) + 0.5 * z * (1.0 - t * t) * c * (1.0 + 3.0 * a * z * z)
    if kind == "silu":
        s = 1.0 / (1.0 + np.exp(-z))
        return s + z * s * (1.0 - s)
    raise ValueError(kind)


def linear_fwd(x, w, b=None, kind="none", res=None):
    """(y, z): z = x w + b, y = act(z) + res."""
    x, w, b, res = _f64(x, w, b, res)
    z = x @ w if b is None else x @ w + b
    y = act(z, kind)
    return (y if res is None else y + res), z


def linear_bwd(dy, x, w, z=None, kind="none"):
    """(dx, dw, db) of linear_fwd with pre-activation z; the residual's gradient is dy."""
    dy, x, w, z = _f64(dy, x, w, z)
    dz = dy if kind == "none" else dy * act_grad(z, kind)
    return dz @ w.T, x.T @ dz, dz.sum(axis=0)


# ------------------------------------------------------- losses of a linear head
def _log_softmax(z):
    top = z.max(axis=1, keepdims=True)
    lse = top[:, 0] + np.log(np.exp(z - top).sum(axis=1))
    return z - lse[:, None], lse


def ce(x, w, labels, ignore=-100, dloss=None, mean=True):
    """Cross entropy of softmax(x w), x [M, K], w [K, V]: dict(loss [M], lse [M], total (sum,
    rows counted), dx, dw).  dloss: the gradient of the mean (or sum) over the counted
    rows (a number), or of each row's loss (an array; mean is then ignored)."""
    x, w = _f64(x, w)
    labels = np.asarray(labels)
    logq, lse = _log_softmax(x @ w)
    on = labels != ignore
    loss = np.zeros(len(x))
    loss[on] = -logq[np.nonzero(on)[0], labels[on]]
    target = np.zeros_like(logq)
    target[np.nonzero(on)[0], labels[on]] = 1.0
    g = _row_scale(on, dloss, mean)
    dz = np.where(on[:, None], np.exp(logq) - target, 0.0) * g[:, None]
    return dict(loss=loss, lse=lse, total=np.array([loss.sum(), on.sum()]), dx=dz @ w.T, dw=x.T @ dz)


def _row_scale(on, dloss, mean):
    if dloss is None:
        dloss = 1.0
    if np.ndim(dloss):
        return np.where(on, np.asarray(dloss, dtype=np.float64), 0.0)
    return np.where(on, float(dloss) / (max(int(on.sum()), 1) if mean else 1), 0.0)


def kd_prob(index, logits, T):
    """softmax(logits / T) over each row's present entries (index >= 0, logit above
    -inf), 0 for the others; a row without any has weights of 0."""
    index, (logits,) = np.asarray(index), _f64(logits)
    t = np.where(index >= 0, logits / T, -np.inf)
    top = t.max(axis=1, keepdims=True)
    e = np.where(np.isneginf(t), 0.0, np.exp(t - np.where(np.isneginf(top), 0.0, top)))
    s = e.sum(axis=1, keepdims=True)
    return np.divide(e, s, out=np.zeros_like(e), where=s > 0)


def kd(x, w, index, logits, T=1.0, dloss=None, mean=True):
    """T^2 sum_j p_j (log p_j - log q_{index_j}) with p = kd_prob and q = softmax(x w / T); an
    index may stand in a row more than once.  The dict of ce, and prob."""
    x, w = _f64(x, w)
    index = np.asarray(index)
    p = kd_prob(index, logits, T)
    logq, lse = _log_softmax(x @ w / T)
    on = p.sum(axis=1) > 0
    target = np.zeros_like(logq)
    loss = np.zeros(len(x))
    for m in np.nonzero(on)[0]:
        for j in np.nonzero(p[m] > 0)[0]:
            target[m, index[m, j]] += p[m, j]
            loss[m] += T * T * p[m, j] * (math.log(p[m, j]) - logq[m, index[m, j]])
    g = _row_scale(on, dloss, mean)
    dz = np.where(on[:, None], np.exp(logq) - target, 0.0) * (T * g)[:, None]
    return dict(loss=loss, lse=lse, total=np.array([loss.sum(), on.sum()]), dx=dz @ w.T, dw=x.T @ dz, prob=p)
