"""Performance cases of the feed-forward operators: a pre-norm feed-forward block
of a language model, dense or with pruned neurons, in training and in serving.

Six operators:

  ln_fwd      layer norm over rows, with the statistics that its gradient needs
  ln_bwd      its gradient: inputs, weight and bias, plus the gradient that the
              residual path brings
  linear_fwd  Y = act(X W^T + bias) + residual over a [N, K] weight matrix
  linear_bwd  dX, dW and dbias of it (dW in binary32 where the optimiser reads it)
  glu_fwd     H = act(X Wg^T + bg) * (X Wu^T + bu), with both pre-activations kept
              for the backward pass when training
  glu_bwd     dX, dWg, dWu, dbg and dbu of it

Widths are powers of two and the 60% of them that filter-wise pruning keeps
(2458 of 4096, 4915 of 8192, 9830 of 16384), so the products are ragged.  A pruned weight matrix has
the pitch that the compaction writes: rows of a multiple of 64 elements, the
padding +0.  Activations are normals as a layer norm leaves them, weights follow
the 1/fan_in law.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda"
EPS = 1e-5
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases
def listed():
    return [
        # the norm of one token of a serving loop: launch latency
        dict(name="ln_fwd_token", op="ln_fwd", rows=1, cols=4096, type="bf16", pitch="packed", affine=True),
        # the norm of a training batch
        dict(name="ln_fwd_16384x4096", op="ln_fwd", rows=16384, cols=4096, type="bf16", pitch="packed", affine=True),
        # a ragged width whose rows start on 4-byte boundaries, no residual gradient
        dict(name="ln_bwd_5000x2458", op="ln_bwd", rows=5000, cols=2458, type="f16", pitch="packed", affine=True,
             residual=False),
        # the norm's gradient of a training batch, joined with the residual path's
        dict(name="ln_bwd_16384x4096", op="ln_bwd", rows=16384, cols=4096, type="bf16", pitch="packed", affine=True,
             residual=True),
        # the down projection of one token, 60% of 16384 neurons kept: reads 80 MB of weights
        dict(name="linear_fwd_token", op="linear_fwd", M=1, K=9830, N=4096, type="bf16", pitch="padded", act="none",
             bias=False, residual=True, keep_z=False),
        # the same projection over a long prompt or a training batch
        dict(name="linear_fwd_8192", op="linear_fwd", M=8192, K=9830, N=4096, type="bf16", pitch="padded", act="none",
             bias=True, residual=True, keep_z=False),
        # a small plain layer with an odd input width in fine-tuning: packed rows of 1229 elements
        dict(name="linear_bwd_256", op="linear_bwd", M=256, K=1229, N=1024, type="f16", pitch="packed", act="gelu",
             bias=True, dw="f16"),
        # the down projection's gradients in training, dW in binary32 for the optimiser
        dict(name="linear_bwd_8192", op="linear_bwd", M=8192, K=9830, N=4096, type="bf16", pitch="padded", act="none",
             bias=True, dw="f32"),
        # sixteen sequences decoded together: both projections of the pruned block, 161 MB of weights
        dict(name="glu_fwd_16", op="glu_fwd", M=16, K=4096, N=9830, type="bf16", pitch="padded", act="silu",
             bias=False, save=False),
        # the block's forward pass over a training batch, pre-activations kept
        dict(name="glu_fwd_8192", op="glu_fwd", M=8192, K=4096, N=9830, type="bf16", pitch="padded", act="silu",
             bias=False, save=True),
        # fine-tuning a small pruned block on a ragged batch
        dict(name="glu_bwd_1000", op="glu_bwd", M=1000, K=1024, N=2458, type="f16", pitch="packed", act="gelu_tanh",
             bias=True),
        # the block's gradients over a training batch
        dict(name="glu_bwd_8192", op="glu_bwd", M=8192, K=4096, N=9830, type="bf16", pitch="padded", act="silu",
             bias=False),
    ]


def _log(rng, lo, hi):
    """Spread over the logarithm of [lo, hi], odd numbers among them."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if n > 256 and rng.random() < 0.6:  # widths are mostly multiples of 64, batches often are
        n = n // 64 * 64
    return n - 1 if n == 3072 else n


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "linear_fwd", "linear_fwd", "linear_bwd", "glu_fwd", "glu_fwd", "glu_bwd"])
    pitch = rng.choice(["packed", "packed", "padded"])
    if op.startswith("ln"):
        rows = _log(rng, 1, 16384)
        c = dict(op=op, rows=rows, cols=min(_log(rng, 64, 16384), 16384 * 4096 // rows),
                 type=rng.choice(["bf16", "f16", "f32"]), pitch=pitch, affine=rng.random() < 0.8)
        if op == "ln_bwd":
            c["residual"] = rng.random() < 0.5
        return c
    while True:
        M, K, N = _log(rng, 1, 8192), _log(rng, 64, 16384), _log(rng, 64, 16384)
        if M * K * N <= 8192 * 4096 * 9830 and K * N <= 8192 * 8192:
            break
    c = dict(op=op, M=M, K=K, N=N, type=rng.choice(["bf16", "bf16", "f16"]), pitch=pitch, bias=rng.random() < 0.5)
    if op.startswith("linear"):
        c["act"] = rng.choice(["none", "none", "relu", "silu", "gelu", "gelu_tanh", "sigmoid"])
        if op == "linear_fwd":
            c.update(residual=rng.random() < 0.5, keep_z=c["act"] != "none" and rng.random() < 0.5)
        else:  # an activation's gradient is rounded to the operands' type, so dW is kept in that type too
            c["dw"] = rng.choice([c["type"], "f32"]) if c["act"] == "none" else c["type"]
        return c
    c["act"] = rng.choice(["silu", "silu", "gelu", "gelu_tanh", "relu", "sigmoid"])
    if op == "glu_fwd":
        c["save"] = rng.random() < 0.5
    return c


def work(c):
    e = 4 if c["type"] == "f32" else 2
    if c["op"] == "ln_fwd":
        n = c["rows"] * c["cols"]
        return {"bytes": 2 * e * n + 8 * c["rows"] + (8 * c["cols"] if c["affine"] else 0), "flops": 8 * n}
    if c["op"] == "ln_bwd":
        n = c["rows"] * c["cols"]
        return {"bytes": (4 if c["residual"] else 3) * e * n + 8 * c["rows"] + (12 if c["affine"] else 8) * c["cols"],
                "flops": 16 * n}
    M, K, N = c["M"], c["K"], c["N"]
    b = 4 * N if c["bias"] else 0
    if c["op"] == "linear_fwd":
        out = 1 + bool(c["residual"]) + bool(c["keep_z"])
        return {"bytes": e * (M * K + N * K + out * M * N) + b, "flops": 2 * M * N * K}
    if c["op"] == "linear_bwd":
        read = M * N * (1 + (c["act"] != "none")) + M * K + N * K
        return {"bytes": e * (read + M * K) + (4 if c["dw"] == "f32" else e) * N * K + b, "flops": 4 * M * N * K}
    if c["op"] == "glu_fwd":
        return {"bytes": e * (M * K + 2 * N * K + (3 if c["save"] else 1) * M * N) + 2 * b, "flops": 4 * M * N * K}
    return {"bytes": e * (3 * M * N + 2 * M * K + 4 * N * K) + 2 * b, "flops": 8 * M * N * K}


# ----------------------------------------------------------------- the inputs
def _rows(c, rows, cols, dtype):
    """A zeroed [rows, cols] matrix with the case's row pitch."""
    ld = cols if c["pitch"] == "packed" else (cols + 63) // 64 * 64
    return torch.zeros(rows, ld, dtype=dtype, device=DEV)[:, :cols]


def _normal(c, g, rows, cols, scale=1.0, shift=0.0):
    x = torch.randn(rows, cols, generator=g, device=DEV, dtype=torch.float32)
    return _rows(c, rows, cols, TYPES[c["type"]]).copy_(x * scale + shift)


def _vector(g, n, scale, shift=0.0):
    return torch.randn(n, generator=g, device=DEV, dtype=torch.float32) * scale + shift


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt, s = TYPES[c["type"]], dict(case=c)
    if c["op"].startswith("ln"):
        R, C = c["rows"], c["cols"]
        # a residual stream: rows of different scales with a mean of their own
        scale, shift = torch.exp(0.5 * _vector(g, R, 1.0))[:, None], 0.3 * _vector(g, R, 1.0)[:, None]
        s["X"] = _normal(c, g, R, C, scale, shift)
        s["gamma"] = _vector(g, C, 0.1, 1.0) if c["affine"] else None
        s["beta"] = _vector(g, C, 0.1) if c["affine"] else None
        if c["op"] == "ln_fwd":
            s.update(Y=_rows(c, R, C, dt), mean=torch.zeros(R, device=DEV), rstd=torch.zeros(R, device=DEV))
            return s
        s["dY"] = _normal(c, g, R, C)
        s["dR"] = _normal(c, g, R, C) if c["residual"] else None
        x = s["X"].double()
        mean = x.mean(1)
        s["mean"] = mean.float()
        s["rstd"] = ((x - mean[:, None]).square().mean(1) + EPS).rsqrt().float()
        s.update(dX=_rows(c, R, C, dt), dgamma=torch.zeros(C, device=DEV), dbeta=torch.zeros(C, device=DEV))
        return s
    M, K, N = c["M"], c["K"], c["N"]
    s["X"] = _normal(c, g, M, K)
    if c["op"].startswith("linear"):
        s["W"] = _normal(c, g, N, K, 1 / math.sqrt(K))
        s["bias"] = _vector(g, N, 0.1) if c["bias"] else None
        if c["op"] == "linear_fwd":
            s["R"] = _normal(c, g, M, N) if c["residual"] else None
            s.update(Y=_rows(c, M, N, dt), Z=_rows(c, M, N, dt) if c["keep_z"] else None)
            return s
        s["dY"] = _normal(c, g, M, N)
        s["Z"] = _normal(c, g, M, N) if c["act"] != "none" else None
        s.update(dX=_rows(c, M, K, dt), dW=_rows(c, N, K, TYPES[c["dw"]]),
                 dbias=torch.zeros(N, device=DEV) if c["bias"] else None)
        return s
    s["Wg"], s["Wu"] = _normal(c, g, N, K, 1 / math.sqrt(K)), _normal(c, g, N, K, 1 / math.sqrt(K))
    s["bg"], s["bu"] = (_vector(g, N, 0.1), _vector(g, N, 0.1)) if c["bias"] else (None, None)
    if c["op"] == "glu_fwd":
        keep = (_rows(c, M, N, dt), _rows(c, M, N, dt)) if c["save"] else (None, None)
        s.update(H=_rows(c, M, N, dt), G=keep[0], U=keep[1])
        return s
    s["dH"], s["G"], s["U"] = (_normal(c, g, M, N) for _ in range(3))
    s.update(dX=_rows(c, M, K, dt), dWg=_rows(c, N, K, dt), dWu=_rows(c, N, K, dt),
             dbg=torch.zeros(N, device=DEV) if c["bias"] else None,
             dbu=torch.zeros(N, device=DEV) if c["bias"] else None)
    return s


# ------------------------------------------------------------- the plain form
def _act(name, z):
    if name == "none":
        return z
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "sigmoid":
        return 1 / (1 + torch.exp(-z))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))


def _dact(name, z):
    """The activation's derivative (0 at the corner of relu)."""
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "sigmoid":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 - p)
    if name == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    t = torch.tanh(a * (z + 0.044715 * z * z * z))
    return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * a * (1 + 3 * 0.044715 * z * z)


def _ln_fwd(s, dt):
    x = s["X"].to(dt)
    mean = x.mean(1)
    rstd = ((x - mean[:, None]).square().mean(1) + EPS).rsqrt()
    y = (x - mean[:, None]) * rstd[:, None]
    return (y if s["gamma"] is None else y * s["gamma"].to(dt) + s["beta"].to(dt)), mean, rstd


def _ln_bwd(s, dt):
    dy, rstd = s["dY"].to(dt), s["rstd"].to(dt)[:, None]
    xn = (s["X"].to(dt) - s["mean"].to(dt)[:, None]) * rstd
    t = dy if s["gamma"] is None else dy * s["gamma"].to(dt)
    dx = rstd * (t - t.mean(1)[:, None] - xn * (t * xn).mean(1)[:, None])
    return (dx if s["dR"] is None else dx + s["dR"].to(dt)), (dy * xn).sum(0), dy.sum(0)


def _linear_fwd(s, dt):
    z = s["X"].to(dt) @ s["W"].to(dt).t()
    z = z if s["bias"] is None else z + s["bias"].to(dt)
    y = _act(s["case"]["act"], z)
    return (y if s["R"] is None else y + s["R"].to(dt)), (z if s["case"]["keep_z"] else None)


def _linear_bwd(s, dt):
    dz = s["dY"].to(dt)
    if s["Z"] is not None:
        dz = dz * _dact(s["case"]["act"], s["Z"].to(dt))
    return dz @ s["W"].to(dt), dz.t() @ s["X"].to(dt), (dz.sum(0) if s["case"]["bias"] else None)


def _glu_fwd(s, dt):
    x, save = s["X"].to(dt), s["case"]["save"]
    g, u = x @ s["Wg"].to(dt).t(), x @ s["Wu"].to(dt).t()
    if s["bg"] is not None:
        g, u = g + s["bg"].to(dt), u + s["bu"].to(dt)
    return _act(s["case"]["act"], g) * u, (g if save else None), (u if save else None)


def _glu_bwd(s, dt):
    dh, g, x, act = s["dH"].to(dt), s["G"].to(dt), s["X"].to(dt), s["case"]["act"]
    dg, du = dh * s["U"].to(dt) * _dact(act, g), dh * _act(act, g)
    b = s["case"]["bias"]
    return (dg @ s["Wg"].to(dt) + du @ s["Wu"].to(dt), dg.t() @ x, du.t() @ x,
            dg.sum(0) if b else None, du.sum(0) if b else None)


PLAIN = {"ln_fwd": _ln_fwd, "ln_bwd": _ln_bwd, "linear_fwd": _linear_fwd, "linear_bwd": _linear_bwd,
         "glu_fwd": _glu_fwd, "glu_bwd": _glu_bwd}
#: the outputs of each operator and the state's buffers that say their types
NAMES = {"ln_fwd": ("Y", "mean", "rstd"), "ln_bwd": ("dX", "dgamma", "dbeta"), "linear_fwd": ("Y", "Z"),
         "linear_bwd": ("dX", "dW", "dbias"), "glu_fwd": ("H", "G", "U"),
         "glu_bwd": ("dX", "dWg", "dWu", "dbg", "dbu")}


# ------------------------------------------------------------------- the pass
def _call(s):
    """One call of the package, into the buffers that the program keeps."""
    import paper_1807_11091_amd as sa
    c = s["case"]
    if c["op"] == "ln_fwd":
        sa.layer_norm_fwd(s["X"], s["gamma"], s["beta"], eps=EPS, Y=s["Y"], mean=s["mean"], rstd=s["rstd"])
    elif c["op"] == "ln_bwd":
        sa.layer_norm_bwd(s["dY"], s["X"], s["mean"], s["rstd"], s["gamma"], dR=s["dR"], dX=s["dX"],
                          dgamma=s["dgamma"], dbeta=s["dbeta"])
    elif c["op"] == "linear_fwd":
        sa.linear_fwd(s["X"], s["W"], s["bias"], R=s["R"], act=sa.ACTS[c["act"]], Y=s["Y"], Z=s["Z"])
    elif c["op"] == "linear_bwd":
        sa.linear_bwd(s["dY"], s["X"], s["W"], Z=s["Z"], act=sa.ACTS[c["act"]], dX=s["dX"], dW=s["dW"],
                      dbias=s["dbias"])
    elif c["op"] == "glu_fwd":
        sa.glu_fwd(s["X"], s["Wg"], s["Wu"], s["bg"], s["bu"], act=sa.ACTS[c["act"]], H=s["H"], G=s["G"], U=s["U"])
    else:
        sa.glu_bwd(s["dH"], s["X"], s["Wg"], s["Wu"], s["G"], s["U"], act=sa.ACTS[c["act"]], dX=s["dX"],
                   dWg=s["dWg"], dWu=s["dWu"], dbg=s["dbg"], dbu=s["dbu"])


def _outputs(c):
    """Names of the case's outputs."""
    left_out = {"linear_fwd": () if c.get("keep_z") else ("Z",), "linear_bwd": () if c.get("bias") else ("dbias",),
                "glu_fwd": () if c.get("save") else ("G", "U"), "glu_bwd": () if c.get("bias") else ("dbg", "dbu")}
    return [n for n in NAMES[c["op"]] if n not in left_out.get(c["op"], ())]


def run(s):
    c = s["case"]
    if own:
        _call(s)
        return {n: s[n] for n in _outputs(c)}
    out = dict(zip(NAMES[c["op"]], PLAIN[c["op"]](s, torch.float32)))
    return {n: out[n].to(s[n].dtype) for n in _outputs(c)}


# ------------------------------------------------- the definitions in 64 bits
def _phi(name, z):
    """Value and derivative of an activation in binary64, from torch's own
    special functions and differentiation."""
    f = {"none": lambda t: t, "relu": torch.relu, "sigmoid": torch.sigmoid, "silu": lambda t: t * torch.sigmoid(t),
         "gelu": lambda t: t * torch.special.ndtr(t),
         "gelu_tanh": lambda t: t * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (t + 0.044715 * t.pow(3)))}[name]
    with torch.enable_grad():
        t = z.detach().requires_grad_(True)
        y = f(t)
        (d,) = torch.autograd.grad(y, t, torch.ones_like(y))
    return y.detach(), d


def exact(c, seed):
    s = prepare(c, seed)
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    op = c["op"]
    if op == "ln_fwd":
        var, mean = torch.var_mean(d["X"], 1, unbiased=False)
        rstd = 1 / torch.sqrt(var + EPS)
        y = torch.addcmul(-mean * rstd, d["X"].t(), rstd).t()
        out = {"Y": torch.addcmul(d["beta"], y, d["gamma"]) if c["affine"] else y, "mean": mean, "rstd": rstd}
    elif op == "ln_bwd":
        n = (d["X"] - d["mean"].unsqueeze(1)).mul_(d["rstd"].unsqueeze(1))
        q = d["dY"] * d["gamma"] if c["affine"] else d["dY"]
        k = c["cols"]
        dx = (q - torch.ones_like(n) * (q.sum(1, keepdim=True) / k) - n * ((q * n).sum(1, keepdim=True) / k))
        dx.mul_(d["rstd"].unsqueeze(1))
        out = {"dX": dx + d["dR"] if c["residual"] else dx, "dgamma": (d["dY"] * n).sum(0), "dbeta": d["dY"].sum(0)}
    elif op == "linear_fwd":
        z = torch.mm(d["W"], d["X"].t()).t()
        z = torch.add(z, d["bias"]) if c["bias"] else z
        y = _phi(c["act"], z)[0]
        out = {"Y": torch.add(d["R"], y) if c["residual"] else y, "Z": z}
    elif op == "linear_bwd":
        dz = d["dY"] if c["act"] == "none" else _phi(c["act"], d["Z"])[1].mul_(d["dY"])
        out = {"dX": torch.mm(d["W"].t(), dz.t()).t(), "dW": torch.mm(d["X"].t(), dz).t(), "dbias": dz.sum(0)}
    elif op == "glu_fwd":
        g, u = torch.mm(d["Wg"], d["X"].t()).t(), torch.mm(d["Wu"], d["X"].t()).t()
        if c["bias"]:
            g, u = torch.add(g, d["bg"]), torch.add(u, d["bu"])
        out = {"H": torch.mul(u, _phi(c["act"], g)[0]), "G": g, "U": u}
    else:
        a, da = _phi(c["act"], d["G"])
        du, dg = a.mul_(d["dH"]), da.mul_(d["U"]).mul_(d["dH"])
        out = {"dX": torch.addmm(torch.mm(dg, d["Wg"]), du, d["Wu"]), "dWg": torch.mm(d["X"].t(), dg).t(),
               "dWu": torch.mm(d["X"].t(), du).t(), "dbg": dg.sum(0), "dbu": du.sum(0)}
    return {n: out[n].contiguous() for n in _outputs(c)}
