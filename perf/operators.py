"""The operators that stand between the layers of a network, each as a user's program calls it, on their own or one pass forward and back.

A case is a dict of plain values.  ``kind`` names the operator:

  dropout   Y = R + dropout(X), R optional; the gradient is the same call on dY
  norm      layer norm, then an activation, then dropout: Y = dropout(act(gamma xhat + beta))
  add_norm  H = R + dropout(X) and Y = gamma xhat(H) + beta, the two steps around a residual connection
  gated     H = act(X W_gate + b_gate) * (X W_up + b_up) with W = [W_gate | W_up]

``step`` adds the backward pass, which returns the gradients of all inputs and weights.  Tensors are fp32, as everywhere in
this library.  Random numbers come from a counter-based generator, Philox4x32 with ten rounds (Salmon, Moraes, Dror and
Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011), whose seed and step are inputs: element (i, c) takes word
c % 4 of the block with key = seed and counter = (c / 4, i, site, step), and is dropped where that word is below p 2^32.
The sizes are those of the graphs and widths in this repository's benchmark and tests.
"""
import functools
import math

import numpy as np
import torch

own = False

EPS = 1e-5
SITE = 3                             # which dropout of a network this one is
ELU, RELU, NONE = "elu", "relu", "none"


def listed():
    return [
        # attention coefficients or hidden features of a citation graph's training step: the launch is what it costs
        dict(name="dropout_small", kind="dropout", n=2048, f=16, p=0.6, residual=False),
        # the end of a residual block on a million nodes: two arrays in, one out
        dict(name="dropout_residual", kind="dropout", n=1 << 20, f=256, p=0.1, residual=True),
        # inference or the forward half on a small graph, sizes that are multiples of nothing, ReLU as in deep convolution nets
        dict(name="norm_ragged_forward", kind="norm", n=3001, f=203, act=RELU, p=0.5, step=False),
        # 47 classes' worth of columns on a mid-sized graph, no dropout: rows of less than a wavefront
        dict(name="norm_narrow_step", kind="norm", n=1 << 17, f=47, act=NONE, p=0.0, step=True),
        # a hidden layer of a network on a million nodes: norm, activation and dropout in training
        dict(name="norm_wide_step", kind="norm", n=1 << 20, f=256, act=ELU, p=0.5, step=True),
        # around the attention layer of a small graph
        dict(name="add_norm_small_step", kind="add_norm", n=2708, f=64, p=0.1, step=True),
        # the same on a large one, features of eight heads of 64
        dict(name="add_norm_step", kind="add_norm", n=1 << 18, f=512, p=0.1, step=True),
        # one node is asked for: the weights are all there is to read
        dict(name="gated_single", kind="gated", n=1, f_in=256, f_out=512, gate="silu", bias=True, keep=False, step=False),
        # inference on a small graph, odd widths
        dict(name="gated_ragged_forward", kind="gated", n=3001, f_in=203, f_out=259, gate="gelu", bias=True, keep=False,
             step=False),
        # a training step on a small graph, narrow
        dict(name="gated_small_step", kind="gated", n=2708, f_in=64, f_out=128, gate="silu", bias=True, keep=True, step=True),
        # a block after the attention layer of a mid-sized graph; the projections are formed again in backward
        dict(name="gated_lean_step", kind="gated", n=1 << 17, f_in=128, f_out=256, gate="sigmoid", bias=False, keep=False,
             step=True),
        # the largest: 512 features and four times that in between, two of them gated away
        dict(name="gated_wide_step", kind="gated", n=1 << 16, f_in=512, f_out=1024, gate="silu", bias=True, keep=True,
             step=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A feature width: half of them multiples of 16, the others any number."""
    w = _log_int(rng, lo, hi)
    return max(16, w // 16 * 16) if rng.random() < 0.5 else w


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["dropout", "norm", "norm", "add_norm", "gated", "gated", "gated"])
        c = dict(kind=kind)
        if kind == "gated":
            c.update(n=_log_int(rng, 1, 1 << 18), f_in=_width(rng, 16, 512), f_out=_width(rng, 7, 1024),
                     gate=rng.choice(["sigmoid", "silu", "gelu"]), bias=rng.random() < 0.5, keep=rng.random() < 0.5,
                     step=rng.random() < 0.7)
        else:
            c.update(n=_log_int(rng, 300, 1 << 20), f=_width(rng, 7, 1024), p=rng.choice([0.1, 0.2, 0.5, 0.6]))
            if kind == "dropout":
                c.update(residual=rng.random() < 0.5)
            elif kind == "norm":
                c.update(step=rng.random() < 0.7)
                # a ReLU whose input is within rounding of zero falls on either side, which changes a gradient by its full
                # size: backward is drawn with the smooth activations
                c.update(act=rng.choice([NONE, ELU] if c["step"] else [NONE, ELU, RELU]))
                if rng.random() < 0.3:
                    c.update(p=0.0)
            else:
                c.update(step=rng.random() < 0.7)
        if _cost(c) <= most and c["n"] * c.get("f", 1) <= 1 << 28:
            return c


# ---- sizes ---------------------------------------------------------------------------------------
def work(case):
    """Each input read once and each output written once; the multiplications and additions of the formulas."""
    n, kind = case["n"], case["kind"]
    if kind == "gated":
        m, k = case["f_in"], case["f_out"]
        weights = 2 * k * (m + (1 if case["bias"] else 0))
        if not case["step"]:
            return {"bytes": 4.0 * (n * m + weights + n * k), "flops": 4.0 * n * m * k}
        return {"bytes": 4.0 * (2 * n * m + 2 * weights + 2 * n * k), "flops": 12.0 * n * m * k}
    f = case["f"]
    if kind == "dropout":
        return {"bytes": 4.0 * n * f * (3 if case["residual"] else 2), "flops": 2.0 * n * f}
    arrays = 2 if kind == "norm" else 4                    # X, Y / X, R, H, Y
    if not case["step"]:
        return {"bytes": 4.0 * (arrays * n * f + 2 * f + 2 * n), "flops": 8.0 * n * f}
    arrays += 2 if kind == "norm" else 4                   # dY, dX / dY, dH, dR, dX
    return {"bytes": 4.0 * (arrays * n * f + 4 * f + 2 * n), "flops": 24.0 * n * f}


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 150e12


# ---- inputs --------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    s = dict(case)
    n = case["n"]
    if case["kind"] == "gated":
        m, k = case["f_in"], case["f_out"]
        s["X"] = normal(n, m)
        s["W"] = normal(m, 2 * k) / math.sqrt(m)
        s["b"] = normal(2 * k) * 0.1 if case["bias"] else None
        if case["step"]:
            s["dH"] = normal(n, k)
        return s
    f = case["f"]
    # what a layer leaves: columns of their own scale and offset
    s["X"] = normal(n, f) * (0.5 + torch.rand(f, generator=gen, device="cuda")) + 0.3 * normal(f)
    if case["kind"] == "add_norm" or case.get("residual"):
        s["R"] = normal(n, f)
    if case["kind"] != "dropout":
        s["gamma"], s["beta"] = 1.0 + 0.1 * normal(f), 0.1 * normal(f)
        if case["step"]:
            s["dY"] = normal(n, f)
            if case["kind"] == "add_norm":
                s["dH"] = normal(n, f)
    # {seed, step} of the generator, on the device: a program adds one to the step after every training step
    s["rng"] = torch.randint(0, 1 << 62, (2,), generator=gen, device="cuda", dtype=torch.int64)
    s["rng"][1] &= (1 << 20) - 1
    return s


# ---- one pass ------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own_pass(s)
    return {"dropout": _dropout_pass, "norm": _norm_pass, "add_norm": _add_norm_pass, "gated": _gated_pass}[s["kind"]](s)


_M32 = 0xFFFFFFFF


def _round(block, _):
    c0, c1, c2, c3, k0, k1 = block
    a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                # 64 bits of each product; int64 wraps
    return ((b >> 32) & _M32) ^ c1 ^ k0, b & _M32, ((a >> 32) & _M32) ^ c3 ^ k1, a & _M32, \
        (k0 + 0x9E3779B9) & _M32, (k1 + 0xBB67AE85) & _M32


def _kept(s, n, f):
    """Which elements of an [n, f] array stay."""
    seed, step = s["rng"][0], s["rng"][1]
    col = torch.arange((f + 3) // 4, device="cuda").expand(n, -1)
    row = torch.arange(n, device="cuda")[:, None]
    start = (col, row, torch.full_like(row, SITE), step & _M32, seed & _M32, (seed >> 32) & _M32)
    words = functools.reduce(_round, range(10), start)[:4]
    words = torch.stack(words, dim=-1).reshape(n, -1)[:, :f]
    return words >= int(round(float(np.float32(s["p"])) * 2.0 ** 32))


def _drop(s, *arrays):
    """Each of the arrays with the same elements dropped and the others scaled."""
    if s["p"] == 0.0:
        return arrays
    kept, scale = _kept(s, *arrays[0].shape), 1.0 / (1.0 - float(np.float32(s["p"])))
    return tuple(torch.where(kept, a * scale, 0.0) for a in arrays)


def _dropout_pass(s):
    y, = _drop(s, s["X"])
    return y + s["R"] if s["residual"] else y


def _normalised(x):
    x = x - x.mean(1, keepdim=True)
    rstd = 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + EPS)
    return x * rstd, rstd


def _norm_gradient(s, xhat, rstd, dz):
    g = dz * s["gamma"]
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    return dx, (dz * xhat).sum(0), dz.sum(0)


def _norm_pass(s):
    xhat, rstd = _normalised(s["X"])
    z = xhat * s["gamma"] + s["beta"]
    a = {NONE: lambda: z, RELU: lambda: z.clamp(min=0.0), ELU: lambda: torch.where(z > 0, z, torch.expm1(z))}[s["act"]]()
    if not s["step"]:
        return _drop(s, a)[0]
    y, da = _drop(s, a, s["dY"])
    dx, dgamma, dbeta = _norm_gradient(s, xhat, rstd, da * torch.exp(z.clamp(max=0.0)) if s["act"] == ELU else da)
    return {"Y": y, "dX": dx, "dgamma": dgamma, "dbeta": dbeta}


def _add_norm_pass(s):
    h = s["R"] + _drop(s, s["X"])[0]
    xhat, rstd = _normalised(h)
    y = xhat * s["gamma"] + s["beta"]
    if not s["step"]:
        return {"H": h, "Y": y}
    dx, dgamma, dbeta = _norm_gradient(s, xhat, rstd, s["dY"])
    dr = s["dH"] + dx
    return {"H": h, "Y": y, "dR": dr, "dX": _drop(s, dr)[0], "dgamma": dgamma, "dbeta": dbeta}


def _gate(kind, a):
    """The activation and its derivative."""
    if kind == "gelu":
        below = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
        return a * below, below + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    g = 1.0 / (1.0 + torch.exp(-a))
    if kind == "silu":
        return a * g, g * (1.0 + a * (1.0 - g))
    return g, g * (1.0 - g)


def _gated_pass(s):
    z = s["X"] @ s["W"]
    if s["bias"]:
        z = z + s["b"]
    a, u = z[:, :s["f_out"]], z[:, s["f_out"]:]
    g, dg = _gate(s["gate"], a)
    if not s["step"]:
        return g * u
    d = torch.cat([s["dH"] * u * dg, s["dH"] * g], dim=1)
    out = {"H": g * u, "dX": d @ s["W"].t(), "dW": s["X"].t() @ d}
    return {**out, "db": d.sum(0)} if s["bias"] else out


# ---- the library's calls ---------------------------------------------------------------------------
def _kept_buffers(s, B):
    """Outputs and scratch that a training loop allocates once and keeps."""
    if "out" in s:
        return s["out"], s["ws"]
    new = functools.partial(torch.empty, dtype=torch.float32, device="cuda")
    n, nbytes = s["n"], 0
    if s["kind"] == "gated":
        m, k = s["f_in"], s["f_out"]
        out = {"H": new(n, k)}
        nbytes = B.gnn_gated_workspace_bytes(False, n, m, k)
        if s["step"]:
            out.update(dX=new(n, m), dW=new(m, 2 * k))
            if s["bias"]:
                out.update(db=new(2 * k))
            nbytes = max(nbytes, B.gnn_gated_workspace_bytes(True, n, m, k))
            s["Z"] = new(n, 2 * k) if s["keep"] else None
    else:
        f = s["f"]
        out = {"Y": new(n, f)}
        if s["kind"] != "dropout":
            s["stat"] = new(n, 2)
            if s["kind"] == "add_norm":
                out.update(H=new(n, f))
            if s["step"]:
                out.update(dX=new(n, f), dgamma=new(f), dbeta=new(f))
                if s["kind"] == "add_norm":
                    out.update(dR=new(n, f))
                nbytes = B.gnn_layer_norm_workspace_bytes(n, f)
    s["out"], s["ws"] = out, B.alloc(nbytes)
    return s["out"], s["ws"]


def _own_pass(s):
    from paper_2308_12093_amd import binding as B

    o, ws = _kept_buffers(s, B)
    n, kind = s["n"], s["kind"]
    if kind == "gated":
        gate = {"sigmoid": B.GNN_GATE_SIGMOID, "silu": B.GNN_GATE_SILU, "gelu": B.GNN_GATE_GELU}[s["gate"]]
        m, k = s["f_in"], s["f_out"]
        if not s["step"]:
            B.gnn_gated_fwd(gate, n, m, k, s["X"], s["W"], s["b"], o["H"], None, ws)
            return o["H"]
        B.gnn_gated_fwd(gate, n, m, k, s["X"], s["W"], s["b"], o["H"], s["Z"], ws)
        B.gnn_gated_bwd(gate, n, m, k, s["X"], s["W"], s["b"], s["Z"], s["dH"], o["dW"], o.get("db"), o["dX"], ws)
        return o
    f = s["f"]
    drop = B.Dropout(s["p"], s["rng"], SITE) if s["p"] > 0.0 else None
    if kind == "dropout":
        B.gnn_dropout(n, f, s["X"], s.get("R"), drop, o["Y"])
        return o["Y"]
    if kind == "norm":
        act = {NONE: B.GNN_ACT_NONE, RELU: B.GNN_ACT_RELU, ELU: B.GNN_ACT_ELU}[s["act"]]
        B.gnn_layer_norm_fwd(n, f, s["X"], s["gamma"], s["beta"], EPS, act, drop, o["Y"], s["stat"])
        if not s["step"]:
            return o["Y"]
        B.gnn_layer_norm_bwd(n, f, s["X"], s["stat"], s["gamma"], s["beta"], act, drop, s["dY"], o["dX"], o["dgamma"],
                             o["dbeta"], ws)
        return o
    B.gnn_add_layer_norm_fwd(n, f, s["X"], s["R"], drop, s["gamma"], s["beta"], EPS, o["H"], o["Y"], s["stat"])
    if s["step"]:
        B.gnn_add_layer_norm_bwd(n, f, o["H"], s["stat"], s["gamma"], drop, s["dY"], s["dH"], o["dR"], o["dX"], o["dgamma"],
                                 o["dbeta"], ws)
    return o


# ---- the definition in 64 bits -----------------------------------------------------------------------
def _times(x, constant):
    """The high and the low 32 bits of x times a 32-bit constant, x in [0, 2^32): by halves of 16 bits, nothing wraps."""
    xl, xh, cl, ch = x % 65536, x // 65536, constant % 65536, constant // 65536
    low, middle = xl * cl, xl * ch + xh * cl
    total = low // 65536 + middle
    return xh * ch + total // 65536, (total % 65536) * 65536 + low % 65536


def _exact_factor(s, n, f):
    """0 for a dropped element, 1 / (1 - p) for the others."""
    p = float(np.float32(s["p"]))
    if p == 0.0:
        return 1.0
    seed, step = (int(v) % (1 << 64) for v in s["rng"].tolist())
    groups = -(-f // 4)
    words = torch.empty(n, 4 * groups, dtype=torch.int64, device="cuda")
    for first in range(0, n, 1 << 17):                     # so that the temporaries stay small
        rows = torch.arange(first, min(n, first + (1 << 17)), device="cuda", dtype=torch.int64)
        x = [torch.arange(groups, device="cuda").repeat(rows.numel()), rows.repeat_interleave(groups)]
        x += [torch.full_like(x[0], SITE), torch.full_like(x[0], step % (1 << 32))]
        key = [seed % (1 << 32), seed // (1 << 32)]
        for _ in range(10):
            h0, l0 = _times(x[0], 0xD2511F53)
            h1, l1 = _times(x[2], 0xCD9E8D57)
            x = [h1.bitwise_xor(x[1]).bitwise_xor(key[0]), l1, h0.bitwise_xor(x[3]).bitwise_xor(key[1]), l0]
            key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
        for w in range(4):
            words[first:first + rows.numel(), w::4] = x[w].view(-1, groups)
    dropped = words[:, :f] < round(p * 4294967296.0)
    return (~dropped).double() / (1.0 - p)


def exact(case, seed):
    s = prepare(case, seed)
    n = case["n"]
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v) and v.is_floating_point()}
    if case["kind"] == "gated":
        k = case["f_out"]
        bias = d.get("b", torch.zeros(2 * k, dtype=torch.float64, device="cuda"))
        a = torch.addmm(bias[:k], d["X"], d["W"][:, :k].contiguous())
        u = torch.addmm(bias[k:], d["X"], d["W"][:, k:].contiguous())
        if case["gate"] == "gelu":                         # a times the normal distribution's integral up to a
            integral = torch.special.ndtr(a)
            act, slope = a * integral, integral + a * torch.exp(-a ** 2 / 2) / math.sqrt(2 * math.pi)
        else:
            sig = torch.sigmoid(a)
            act = sig * a if case["gate"] == "silu" else sig
            slope = sig + act * torch.sigmoid(-a) if case["gate"] == "silu" else sig * torch.sigmoid(-a)
        if not case["step"]:
            return act * u
        da, du = d["dH"] * u * slope, d["dH"] * act
        out = {"H": act * u, "dX": da @ d["W"][:, :k].t() + du @ d["W"][:, k:].t(),
               "dW": torch.cat([d["X"].t() @ da, d["X"].t() @ du], 1)}
        if case["bias"]:
            out["db"] = torch.cat([da.sum(0), du.sum(0)])
        return out
    f = case["f"]
    factor = _exact_factor(s, n, f)
    if case["kind"] == "dropout":
        return d["X"] * factor + d.get("R", 0.0)
    h = d["X"] if case["kind"] == "norm" else d["R"] + factor * d["X"]
    var, mean = torch.var_mean(h, dim=1, correction=0, keepdim=True)
    sigma = (var + EPS).sqrt()
    xhat = (h - mean) / sigma
    y = d["beta"] + d["gamma"] * xhat
    slope = 1.0
    if case["kind"] == "norm":
        if case["act"] == RELU:
            y, slope = y.relu(), (y > 0).double()
        elif case["act"] == ELU:
            slope = y.minimum(torch.zeros_like(y)).exp()
            y = y.relu() + slope - 1.0
        y = y * factor
    if not case["step"]:
        return y if case["kind"] == "norm" else {"H": h, "Y": y}
    dz = d["dY"] * slope * (factor if case["kind"] == "norm" else 1.0)
    out = {"Y": y, "dgamma": (dz * xhat).sum(0), "dbeta": dz.sum(0)}
    # the Jacobian of xhat: (1 - 1 1^T / f - xhat xhat^T / f) / sigma
    g = dz * d["gamma"]
    dh = (g - (g.sum(1, keepdim=True) + xhat * (xhat * g).sum(1, keepdim=True)) / f) / sigma
    if case["kind"] == "norm":
        return {**out, "dX": dh}
    dr = d["dH"] + dh
    return {**out, "H": h, "dR": dr, "dX": dr * factor}
