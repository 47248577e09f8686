"""The operators around attention that a fine-tuning step needs, as timed calls.

  norm    layer norm: forward, and backward with the gradients of weight and bias
  linear  act(x w + bias) + residual: forward and backward, or the forward alone
          for a few tokens (serving)
  mlp     two of them in a row, the activation between: a block's feed-forward part
  ce      softmax cross entropy of a linear head over the vocabulary, with its
          gradients, no logits kept
  kd      distillation from a teacher's top logits on the same head, with its gradients

`own` False: elementary torch operations in 32 bits, rounded to the storage type
once at the end of an operator.  `own` True: the library's calls.
"""
import math

import torch

own = False

DEVICE = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------- the cases
def _norm(name, M, N, dtype):
    return _named(name, dict(kind="norm", M=M, N=N, dtype=dtype))


def _linear(name, M, K, N, dtype, act, bias=True, residual=True, train=True):
    return _named(name, dict(kind="linear", M=M, K=K, N=N, dtype=dtype, act=act, bias=bias, residual=residual, train=train))


def _mlp(name, M, K, N, dtype, act):
    return _named(name, dict(kind="mlp", M=M, K=K, N=N, dtype=dtype, act=act))


def _ce(name, M, K, V, dtype, table, ignored):
    return _named(name, dict(kind="ce", M=M, K=K, V=V, dtype=dtype, table=table, ignored=ignored))


def _kd(name, M, K, V, top, dtype, table, T, absent):
    return _named(name, dict(kind="kd", M=M, K=K, V=V, top=top, dtype=dtype, table=table, T=T, absent=absent))


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # the smallest norm: a toy model kept in fp32 (unit tests, debugging runs); launches and latency
        _norm("norm_tiny_f32", 32, 256, "f32"),
        # an encoder batch of short sentences, BERT-base-like: 8 x 128 tokens of hidden size 768
        _norm("norm_bert", 1024, 768, "bf16"),
        # a packed batch whose hidden size fills no vector load
        _norm("norm_odd", 4099, 1001, "bf16"),
        # the largest norm: 16384 tokens of hidden size 4096, Llama-7B-like
        _norm("norm_wide", 16384, 4096, "bf16"),
        # serving: one token through a fused QKV projection with bias, hidden size 4096
        _linear("linear_one_token", 1, 4096, 12288, "bf16", "none", residual=False, train=False),
        # a GELU layer with bias and residual kept in fp32, a token count that fills no tile
        _linear("linear_f32_ragged", 333, 768, 2304, "f32", "gelu"),
        # the feed-forward part of a block of hidden size 2048, 4096 tokens, the benchmark's projection sizes
        _mlp("mlp_2048_8192", 4096, 2048, 8192, "bf16", "gelu_tanh"),
        # the smallest loss: a toy model in fp32 with a vocabulary of a thousand
        _ce("ce_tiny_f32", 64, 128, 1000, "f32", False, 0.1),
        # a tied embedding table of odd length, 4 x 1024 tokens, GPT-2-medium-like, a tenth of the labels padding
        _ce("ce_tied", 4096, 1024, 50257, "bf16", True, 0.1),
        # the largest loss by hidden size: an untied head, 4096 tokens, Llama-7B-like
        _ce("ce_llama7b", 4096, 4096, 32000, "bf16", False, 0.0),
        # distillation of a toy model in fp32: ragged everything, rows with few or no teacher entries
        _kd("kd_f32_ragged", 250, 500, 5003, 8, "f32", True, 2.0, 0.2),
        # distillation over a vocabulary of 128256 from 32 teacher logits a token, Llama-3.2-1B-like hidden size
        _kd("kd_large_vocab", 2048, 2048, 128256, 32, "bf16", True, 1.0, 0.0),
    ]


ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    kind = rng.choice(["norm", "norm", "linear", "linear", "few", "mlp", "ce", "ce", "kd", "kd"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    f32 = dtype == "f32"
    step = 1 if f32 else 8  # bf16 products have rows of whole 16-byte chunks
    while True:
        if kind == "norm":
            c = _norm("", _log(rng, 1, 32768), rng.choice([1, 8, 64]) * _log(rng, 1, 256), dtype)
            if 32 <= c["M"] * c["N"] <= 1 << 25:
                return c
        elif kind == "few":
            return _linear("", _log(rng, 1, 32), step * _log(rng, 64 // step, 8192 // step),
                           step * _log(rng, 64 // step, 8192 // step), dtype, rng.choice(ACTS), rng.random() < 0.7,
                           rng.random() < 0.5, train=False)
        elif kind == "linear":
            c = _linear("", _log(rng, 1, 8192), step * _log(rng, 64 // step, 4096 // step),
                        step * _log(rng, 64 // step, 8192 // step), dtype, rng.choice(ACTS), rng.random() < 0.7,
                        rng.random() < 0.5)
            if 6.0 * c["M"] * c["K"] * c["N"] <= (2e10 if f32 else 4e11):
                return c
        elif kind == "mlp":
            K = step * _log(rng, 64 // step, 2048 // step)
            c = _mlp("", _log(rng, 1, 4096), K, 4 * K, dtype, rng.choice(ACTS[1:]))
            if 12.0 * c["M"] * c["K"] * c["N"] <= (2e10 if f32 else 4e11):
                return c
        else:
            table = rng.random() < 0.5
            V = _log(rng, 64, 16384 if f32 else 131072)
            if not table and not f32:
                V = (V + 7) // 8 * 8
            M, K = _log(rng, 1, 4096), step * _log(rng, 64 // step, 4096 // step)
            lost = rng.choice([0.0, 0.1, 0.5])
            c = (_ce("", M, K, V, dtype, table, lost) if kind == "ce" else
                 _kd("", M, K, V, rng.choice([1, 5, 8, 20, 32, 50]), dtype, table, rng.choice([1.0, 2.0, 4.0]), lost))
            if 6.0 * M * K * V <= (2e10 if f32 else 1e12):
                return c


# ------------------------------------------------------------------ the inputs
def _randn(gen, shape, dtype, scale=1.0, shift=0.0):
    x = torch.randn(shape, generator=gen, device=DEVICE, dtype=torch.float32)
    return (x * scale + shift).to(dtype)


def _inputs(case, seed):
    """The inputs alone: activations and their gradients ~ N(0, 1), weights ~ N(0, 1 / fan-in), norm weights
    around one.  The head's logits have a deviation of 2, and for half of the tokens the label (the teacher's first
    entry) stands out, as a model's that has learned something does."""
    c = case
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    if c["kind"] == "norm":
        M, N = c["M"], c["N"]
        return {"x": _randn(gen, (M, N), dt, 1.5, 0.3), "weight": _randn(gen, (N,), dt, 0.2, 1.0),
                "bias": _randn(gen, (N,), dt, 0.2), "dy": _randn(gen, (M, N), dt)}
    if c["kind"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        return {"x": _randn(gen, (M, K), dt), "w": _randn(gen, (K, N), dt, K ** -0.5),
                "bias": _randn(gen, (N,), dt, 0.2) if c["bias"] else None,
                "residual": _randn(gen, (M, N), dt) if c["residual"] else None, "dy": _randn(gen, (M, N), dt)}
    if c["kind"] == "mlp":
        M, K, N = c["M"], c["K"], c["N"]
        return {"x": _randn(gen, (M, K), dt), "w1": _randn(gen, (K, N), dt, K ** -0.5), "b1": _randn(gen, (N,), dt, 0.2),
                "w2": _randn(gen, (N, K), dt, N ** -0.5), "b2": _randn(gen, (K,), dt, 0.2),
                "residual": _randn(gen, (M, K), dt), "dy": _randn(gen, (M, K), dt)}
    M, K, V = c["M"], c["K"], c["V"]
    w = _randn(gen, (V, K) if c["table"] else (K, V), dt, 2.0 * K ** -0.5)
    w = w.t() if c["table"] else w  # [K, V]; the table is read as it is stored
    s = {"w": w, "dloss": torch.rand((), generator=gen, device=DEVICE) + 0.5}
    if c["kind"] == "ce":
        first = torch.randint(0, V, (M,), generator=gen, device=DEVICE)
        s["labels"] = torch.where(torch.rand(M, generator=gen, device=DEVICE) < c["ignored"], -100, first)
    else:
        k = c["top"]
        gaps = torch.randint(1, max(2, V // k + 1), (M, k), generator=gen, device=DEVICE)
        s["index"] = (torch.randint(0, V, (M, 1), generator=gen, device=DEVICE) + gaps.cumsum(1)) % V
        s["logits"] = _randn(gen, (M, k), dt, 2.0, 8.0).sort(dim=1, descending=True).values
        first = s["index"][:, 0].clone()
        # some rows have fewer entries, some none (padding)
        lost = torch.rand(M, 1, generator=gen, device=DEVICE) < c["absent"]
        keep = torch.randint(0, k + 1, (M, 1), generator=gen, device=DEVICE)
        s["index"][lost & (torch.arange(k, device=DEVICE) >= keep)] = -1
    known = (torch.rand(M, 1, generator=gen, device=DEVICE) < 0.5).float()
    x = torch.randn((M, K), generator=gen, device=DEVICE)
    s["x"] = (x + 2.0 * known * w.t()[first].float()).to(dt)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["case"] = c = case
    new = lambda *shape, dtype=DTYPES[c["dtype"]]: torch.empty(shape, dtype=dtype, device=DEVICE)
    f32 = torch.float32
    # buffers that a training or serving program keeps from step to step
    if c["kind"] == "norm":
        M, N = c["M"], c["N"]
        s.update(y=new(M, N), mean=new(M, dtype=f32), rstd=new(M, dtype=f32), dx=new(M, N), dweight=new(N), dbias=new(N))
    elif c["kind"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        s["y"] = new(M, N)
        s["z"] = new(M, N) if c["train"] and c["act"] != "none" else None
        if c["train"]:
            s.update(dx=new(M, K), dw=new(K, N), db=new(N) if c["bias"] else None)
    elif c["kind"] == "mlp":
        for k in ("x", "w1", "b1", "w2", "b2", "residual"):
            s[k].requires_grad_(True)
    else:
        M, K = c["M"], c["K"]
        s.update(loss=new(M, dtype=f32), lse=new(M, dtype=f32), total=new(2, dtype=f32), dx=new(M, K),
                 dw=torch.empty_like(s["w"]))
        if c["kind"] == "kd":
            s["prob"] = new(M, c["top"], dtype=f32)
    if own:
        from paper_2607_21624_amd import fbl
        ws = 0
        if c["kind"] == "norm":
            ws = fbl.layer_norm_bwd_workspace(s["x"])
        elif c["kind"] == "linear" and c["train"]:
            ws = fbl.linear_bwd_workspace(s["x"], s["w"])
        elif c["kind"] in ("ce", "kd"):
            ws = fbl.linear_loss_workspace(s["x"], s["w"], c.get("top", 1))
        s["workspace"] = torch.empty(ws, dtype=torch.uint8, device=DEVICE)
    return s


# --------------------------------------------------------------------- one pass
def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_own(s):
    from paper_2607_21624_amd import autograd as ag
    from paper_2607_21624_amd import fbl
    c = s["case"]
    if c["kind"] == "norm":
        y, mean, rstd = fbl.layer_norm_fwd(s["x"], s["weight"], s["bias"], EPS, out=s["y"], mean=s["mean"], rstd=s["rstd"])
        dx, dw, db = fbl.layer_norm_bwd(s["dy"], s["x"], mean, rstd, s["weight"], dx=s["dx"], dweight=s["dweight"],
                                        dbias=s["dbias"], workspace=s["workspace"])
        return y, dx, dw, db
    if c["kind"] == "linear":
        y = fbl.linear_fwd(s["x"], s["w"], s["bias"], c["act"], s["residual"], out=s["y"], z=s["z"])
        if not c["train"]:
            return y
        dx, dw, db = fbl.linear_bwd(s["dy"], s["x"], s["w"], s["z"], c["act"], dx=s["dx"], dw=s["dw"], dbias=s["db"],
                                    workspace=s["workspace"])
        return (y, dx, dw, db) if c["bias"] else (y, dx, dw)
    if c["kind"] == "mlp":
        p = tuple(s[k] for k in ("x", "w1", "b1", "w2", "b2", "residual"))
        y = ag.mlp(*p[:5], act=c["act"], residual=p[5])
        return (y.detach(),) + torch.autograd.grad(y, p, s["dy"])
    if c["kind"] == "ce":
        fbl.linear_ce_fwd(s["x"], s["w"], s["labels"], loss=s["loss"], lse=s["lse"], total=s["total"],
                          workspace=s["workspace"])
        fbl.linear_ce_bwd(s["dloss"], s["x"], s["w"], s["labels"], s["lse"], total=s["total"], dx=s["dx"], dw=s["dw"],
                          workspace=s["workspace"])
    else:
        fbl.linear_kd_fwd(s["x"], s["w"], s["index"], s["logits"], c["T"], loss=s["loss"], lse=s["lse"], prob=s["prob"],
                          total=s["total"], workspace=s["workspace"])
        fbl.linear_kd_bwd(s["dloss"], s["x"], s["w"], s["index"], s["prob"], s["lse"], c["T"], total=s["total"],
                          dx=s["dx"], dw=s["dw"], workspace=s["workspace"])
    return s["loss"], s["lse"], s["total"], s["dx"], s["dw"]


def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        sg = torch.sigmoid(z)
        return sg * (1 + z * (1 - sg))
    return torch.ones_like(z)


def _plain_linear(x, w, bias, act, residual):
    z = x.float() @ w.float()
    if bias is not None:
        z = z + bias.float()
    y = _act(z, act)
    if residual is not None:
        y = y + residual.float()
    return y, z


def _run_plain(s):
    c = s["case"]
    dt = s["x"].dtype
    if c["kind"] == "norm":
        x, w, dy = s["x"].float(), s["weight"].float(), s["dy"].float()
        mean = x.mean(1, keepdim=True)
        xc = x - mean
        rstd = 1.0 / torch.sqrt((xc * xc).mean(1, keepdim=True) + EPS)
        xh = xc * rstd
        g = dy * w
        dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
        return (xh * w + s["bias"].float()).to(dt), dx.to(dt), (dy * xh).sum(0).to(dt), dy.sum(0).to(dt)
    if c["kind"] == "linear":
        y, z = _plain_linear(s["x"], s["w"], s["bias"], c["act"], s["residual"])
        if not c["train"]:
            return y.to(dt)
        dz = s["dy"].float() * _act_grad(z, c["act"])
        out = (y.to(dt), (dz @ s["w"].float().t()).to(dt), (s["x"].float().t() @ dz).to(dt))
        return out + (dz.sum(0).to(dt),) if c["bias"] else out
    if c["kind"] == "mlp":
        x, w1, b1, w2, b2, r = (s[k].detach() for k in ("x", "w1", "b1", "w2", "b2", "residual"))
        h, z = _plain_linear(x, w1, b1, c["act"], None)
        y, _ = _plain_linear(h, w2, b2, "none", r)
        dy = s["dy"].float()
        dz = (dy @ w2.float().t()) * _act_grad(z, c["act"])
        return tuple(t.to(dt) for t in (y, dz @ w1.float().t(), x.float().t() @ dz, dz.sum(0), h.t() @ dy, dy.sum(0), dy))
    x, w = s["x"].float(), s["w"].float()
    M = x.shape[0]
    T = c.get("T", 1.0)
    z = x @ w
    u = z / T if T != 1.0 else z
    top = u.max(1, keepdim=True).values
    lse = (top + torch.log(torch.exp(u - top).sum(1, keepdim=True)))[:, 0]
    if c["kind"] == "ce":
        counted = s["labels"] != -100
        idx = torch.where(counted, s["labels"], 0)[:, None]
        p = counted[:, None].float()
        loss = torch.where(counted, lse - u.gather(1, idx)[:, 0], 0.0)
    else:
        there = s["index"] >= 0
        counted = there.any(1)
        idx = torch.where(there, s["index"], 0)
        t = torch.where(there, s["logits"].float() / T, -math.inf)
        e = torch.where(there, torch.exp(t - t.max(1, keepdim=True).values), 0.0)
        p = e / e.sum(1, keepdim=True).clamp(min=1e-30)
        logp = torch.log(p.clamp(min=1e-38))
        loss = torch.where(counted, T * T * (p * (logp - (u.gather(1, idx) - lse[:, None]))).sum(1), 0.0)
    n = counted.sum().float()
    total = torch.stack([loss.sum(), n])
    g = counted.float() * s["dloss"] / n.clamp(min=1.0) * T
    dz = torch.exp(u - lse[:, None])
    dz.scatter_add_(1, idx, -p)
    dz *= g[:, None]
    dx = (dz @ w.t()).to(dt)
    dw = ((dz.t() @ x).t() if c["table"] else x.t() @ dz).to(dt)
    return loss, lse, total, dx, dw


# -------------------------------------------------------- what it cannot do without
def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    if c["kind"] == "norm":
        M, N = c["M"], c["N"]
        # x read and y written; x and dy read, dx written; weight, bias and their gradients; ~20 operations an element
        return {"bytes": es * (5 * M * N + 4 * N), "flops": 20.0 * M * N}
    if c["kind"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        fwd = M * K + K * N + M * N * (1 + c["residual"])
        if not c["train"]:
            return {"bytes": es * fwd, "flops": 2.0 * M * K * N}
        return {"bytes": es * (fwd + M * N + M * K + K * N), "flops": 6.0 * M * K * N}
    if c["kind"] == "mlp":
        M, K, N = c["M"], c["K"], c["N"]
        # x, residual, dy and the weights read; y, dx and the weights' gradients written
        return {"bytes": es * (5 * M * K + 4 * K * N), "flops": 12.0 * M * K * N}
    M, K, V = c["M"], c["K"], c["V"]
    return {"bytes": es * 2 * (M * K + K * V), "flops": 6.0 * M * K * V}


# ----------------------------------------------------------------- in 64 bits
def exact(case, seed):
    c, s = case, _inputs(case, seed)
    d = {k: v.double() if isinstance(v, torch.Tensor) and v.is_floating_point() else v for k, v in s.items()}
    if c["kind"] == "norm":
        x = d["x"].requires_grad_(True)
        w, b = d["weight"].requires_grad_(True), d["bias"].requires_grad_(True)
        y = (x - x.mean(1, keepdim=True)) / torch.sqrt(x.var(1, unbiased=False, keepdim=True) + EPS) * w + b
        return (y.detach(),) + torch.autograd.grad(y, (x, w, b), d["dy"])
    fn = {"none": lambda t: t, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu,
          "gelu_tanh": lambda t: torch.nn.functional.gelu(t, approximate="tanh")}
    if c["kind"] == "linear":
        leaves = [d["x"].requires_grad_(True), d["w"].requires_grad_(True)]
        z = leaves[0].matmul(leaves[1])
        if c["bias"]:
            leaves.append(d["bias"].requires_grad_(True))
            z = z + leaves[2]
        y = fn[c["act"]](z)
        if c["residual"]:
            y = y + d["residual"]
        return (y.detach(),) + torch.autograd.grad(y, leaves, d["dy"]) if c["train"] else y.detach()
    if c["kind"] == "mlp":
        leaves = [d[k].requires_grad_(True) for k in ("x", "w1", "b1", "w2", "b2", "residual")]
        x, w1, b1, w2, b2, r = leaves
        y = fn[c["act"]](x.matmul(w1) + b1).matmul(w2) + b2 + r
        return (y.detach(),) + torch.autograd.grad(y, leaves, d["dy"])
    x, w, T = d["x"], d["w"], c.get("T", 1.0)
    M, V = x.shape[0], w.shape[1]
    loss, lse = torch.zeros(M, dtype=torch.float64, device=DEVICE), torch.zeros(M, dtype=torch.float64, device=DEVICE)
    if c["kind"] == "ce":
        rows = s["labels"] != -100
    else:
        rows = (s["index"] >= 0).any(1)
    n = rows.sum().double()
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    for m0 in range(0, M, 1024):  # 1024 tokens at a time
        m1 = min(M, m0 + 1024)
        q = torch.log_softmax(x[m0:m1].matmul(w) / T, dim=1)
        lse[m0:m1] = (x[m0:m1].matmul(w[:, 0]) / T) - q[:, 0]
        target = torch.zeros_like(q)
        if c["kind"] == "ce":
            r = rows[m0:m1].nonzero()[:, 0]
            target[r, s["labels"][m0:m1][r]] = 1.0
            loss[m0:m1] = -(target * q).sum(1)
        else:
            for m in rows[m0:m1].nonzero()[:, 0].tolist():
                at = s["index"][m0 + m]
                p = torch.softmax(d["logits"][m0 + m][at >= 0] / T, dim=0)
                loss[m0 + m] = T * T * (p * (torch.log(p) - q[m, at[at >= 0]])).sum()
                target[m].index_add_(0, at[at >= 0], p)
        dz = (torch.exp(q) - target) * (rows[m0:m1, None].double() * T * d["dloss"] / n.clamp(min=1))
        dx[m0:m1] = dz.matmul(w.t())
        dw += x[m0:m1].t().matmul(dz)
    return loss, lse, torch.stack([loss.sum(), n]), dx, dw
