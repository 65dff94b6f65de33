"""The operators of a block that begins with a root-mean-square norm: trained with its activations kept in 8 bits, or served in 8 bits.

A case is a dict of plain values.  ``kind`` names the operator:

  rms      H = X + R (R optional), Y = gamma xhat with xhat = H / sqrt(mean(H^2) + eps); ``step`` adds the backward pass, from H or,
           with ``keep``, from xhat in 8 bits, which forward has written
  kept     an array put into 8 bits, a scale for each row, and read back
  linear   Y = act(X W + b) + R (b, R optional); ``step`` adds the backward pass, from X and X W + b as forward left it (``keep``) or
           formed again
  back     the backward pass of that product from X and X W + b in 8 bits
  linear8  the forward product of rows in 8 bits and weights in 8 bits

Tensors are fp32, as everywhere in this library.  A row x in 8 bits is the integers q = round(x * (127 / max|x|)) (each of the two
operations rounded to a float, ties of the last to even) and the scale max|x| / 127; q stands for q * scale.  xhat has the integers of
H, and the scale of H times 1 / sqrt(mean(H^2) + eps).  Rows of integers are a multiple of 16 bytes apart.  The sizes are those of the
graphs and widths in this repository's benchmark and tests.
"""
import functools
import math

import torch

own = False

EPS = 1e-5
NONE, RELU, ELU, SIGMOID, SILU, GELU = "none", "relu", "elu", "sigmoid", "silu", "gelu"
ACTS = (NONE, RELU, ELU, SIGMOID, SILU, GELU)


def listed():
    return [
        # the beginning of a block on a citation graph, inference: the launch is what it costs
        dict(name="rms_small_forward", kind="rms", n=2708, f=64, residual=True, keep=False, step=False),
        # the first norm of a network: no residual, sizes that are multiples of nothing
        dict(name="rms_ragged_step", kind="rms", n=30011, f=203, residual=False, keep=False, step=True),
        # between two blocks of a large graph, features of eight heads of 64
        dict(name="rms_step", kind="rms", n=1 << 18, f=512, residual=True, keep=False, step=True),
        # the same on a million nodes, where the rows that backward reads are kept in 8 bits
        dict(name="rms_kept_step", kind="rms", n=1 << 20, f=256, residual=True, keep=True, step=True),
        # any other array that backward reads, kept in 8 bits
        dict(name="kept_rows", kind="kept", n=1 << 18, f=512),
        # one node is asked for: the weights are all there is to read
        dict(name="linear_single", kind="linear", n=1, f_in=256, f_out=512, act=SILU, bias=True, residual=False, keep=False,
             step=False),
        # inference on a small graph, odd widths, the end of a residual block
        dict(name="linear_ragged_forward", kind="linear", n=3001, f_in=203, f_out=259, act=GELU, bias=True, residual=True,
             keep=False, step=False),
        # a training step on a mid-sized graph; the projection is formed again in backward
        dict(name="linear_lean_step", kind="linear", n=1 << 17, f_in=128, f_out=256, act=ELU, bias=True, residual=False,
             keep=False, step=True),
        # the largest: 512 features to four times that, what it gives kept for backward
        dict(name="linear_wide_step", kind="linear", n=1 << 16, f_in=512, f_out=2048, act=SILU, bias=True, residual=True,
             keep=True, step=True),
        # the backward half of a step whose activations were kept in 8 bits
        dict(name="linear_kept_back", kind="back", n=1 << 16, f_in=512, f_out=1024, act=SILU, bias=True),
        # one node, served in 8 bits
        dict(name="linear8_single", kind="linear8", n=1, f_in=512, f_out=1024, act=SILU, bias=True, residual=False),
        # every node of a mid-sized graph, served in 8 bits
        dict(name="linear8_wide", kind="linear8", n=1 << 16, f_in=512, f_out=2048, act=SILU, bias=True, residual=True),
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
        kind = rng.choice(["rms", "rms", "kept", "linear", "linear", "back", "linear8"])
        c = dict(kind=kind)
        if kind in ("rms", "kept"):
            c.update(n=_log_int(rng, 1, 1 << 20), f=_width(rng, 7, 6000))
            if kind == "rms":
                c.update(residual=rng.random() < 0.6, step=rng.random() < 0.7)
                c.update(keep=c["step"] and rng.random() < 0.5)
            if c["n"] * c["f"] > 1 << 28:
                continue
        else:
            c.update(n=_log_int(rng, 1, 1 << 18), f_in=_width(rng, 7, 1024), f_out=_width(rng, 7, 2048), bias=rng.random() < 0.6)
            if kind == "linear":
                c.update(residual=rng.random() < 0.5, keep=rng.random() < 0.5, step=rng.random() < 0.6)
                # a ReLU whose input is within rounding of zero falls on either side, which changes a gradient by its full
                # size: backward is drawn with the smooth activations
                c.update(act=rng.choice([a for a in ACTS if a != RELU or not c["step"]]))
            else:
                c.update(act=rng.choice(ACTS))
                if kind == "linear8":
                    c.update(residual=rng.random() < 0.5)
        if _cost(c) <= most:
            return c


# ---- sizes ---------------------------------------------------------------------------------------
def work(case):
    """Each input read once and each output written once; the multiplications and additions of the formulas."""
    n, kind = case["n"], case["kind"]
    if kind == "kept":
        f = case["f"]                                      # X, q, the values
        return {"bytes": 9.0 * n * f + 4.0 * n, "flops": 5.0 * n * f}
    if kind == "rms":
        f, r = case["f"], case["residual"]
        size = 4.0 * ((4 if r else 2) * n * f + f)         # X, R, H, Y / X, Y
        if not case["step"]:
            return {"bytes": size, "flops": 4.0 * n * f}
        kept = 2.0 * n * f + 8.0 * n if case["keep"] else 0.0
        size += 4.0 * ((3 if r else 2) * n * f + 2 * f + 2 * n) + kept      # dY, dH, dR / dY, dX
        return {"bytes": size, "flops": 13.0 * n * f}
    m, k = case["f_in"], case["f_out"]
    weights, y = m * k + (k if case["bias"] else 0), n * k * (2 if case.get("residual") else 1)
    if kind == "linear8":
        return {"bytes": 1.0 * (n * m + m * k) + 4.0 * (n + 2 * k + y), "flops": 2.0 * n * m * k}
    if kind == "back":                                     # X, X W + b, W, dY; dW, db, dX
        return {"bytes": 1.0 * n * (m + k) + 8.0 * n + 4.0 * (m * k + n * k + weights + n * m), "flops": 4.0 * n * m * k}
    if not case["step"]:
        return {"bytes": 4.0 * (n * m + weights + y), "flops": 2.0 * n * m * k}
    return {"bytes": 4.0 * (2 * n * m + 2 * weights + y + n * k), "flops": 6.0 * n * m * k}


def _cost(c):
    w = work(c)
    return w["bytes"] / 4e12 + w["flops"] / 150e12


# ---- inputs --------------------------------------------------------------------------------------
def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    def features(n, f):
        """What a layer leaves: columns of their own scale and offset."""
        return normal(n, f) * (0.5 + torch.rand(f, generator=gen, device="cuda")) + 0.3 * normal(f)

    s = dict(case)
    n, kind = case["n"], case["kind"]
    if kind in ("rms", "kept"):
        f = case["f"]
        s["X"] = features(n, f)
        if kind == "rms":
            s["gamma"] = 1.0 + 0.1 * normal(f)
            if case["residual"]:
                s["R"] = normal(n, f)
            if case["step"]:
                s["dY"] = normal(n, f)
                if case["residual"]:
                    s["dH"] = normal(n, f)
        return s
    m, k = case["f_in"], case["f_out"]
    s["X"] = normal(n, m)                                  # a norm's rows
    s["W"] = normal(m, k) / math.sqrt(m)
    s["b"] = normal(k) * 0.1 if case["bias"] else None
    s["R"] = normal(n, k) if case.get("residual") else None
    if kind == "linear":
        if case["step"]:
            s["dY"] = normal(n, k)
        return s
    s["gamma"] = 1.0 + 0.1 * normal(m)                     # of the norm before: its output is X times this
    s["X8"] = _rows8(s.pop("X"))
    if kind == "linear8":
        s["W8"] = _rows8(s.pop("W").t() * s["gamma"])
    else:
        s["Z8"], s["dY"] = _rows8(features(n, k)), normal(n, k)
    return s


def _rows8(x):
    """x in 8 bits: integers in rows that are a multiple of 16 bytes apart, and a scale for each."""
    top = x.abs().amax(1, keepdim=True).double()
    q = torch.round(x * torch.where(top > 0, 127.0 / top, 0.0).float())
    q = torch.nn.functional.pad(q.to(torch.int8), (0, -x.shape[1] % 16)).contiguous()
    return q, (top / 127.0).float().view(-1)


# ---- one pass ------------------------------------------------------------------------------------
def run(s):
    if own:
        return _own_pass(s)
    return {"rms": _rms_pass, "kept": _kept_pass, "linear": _linear_pass, "back": _back_pass, "linear8": _linear8_pass}[s["kind"]](s)


def _rms_pass(s):
    h = s["X"] + s["R"] if s["residual"] else s["X"]
    rstd = 1.0 / torch.sqrt((h * h).mean(1, keepdim=True) + EPS)
    xhat = h * rstd
    out = {"Y": xhat * s["gamma"]}
    if s["residual"]:
        out.update(H=h)
    if not s["step"]:
        return out
    if s["keep"]:
        q, scale = _rows8(h)
        xhat = q[:, :s["f"]].float() * (scale.view(-1, 1) * rstd)
    g = s["dY"] * s["gamma"]
    dr = rstd * (g - xhat * (g * xhat).mean(1, keepdim=True))
    return {**out, "dR": dr + s["dH"] if s["residual"] else dr, "dgamma": (s["dY"] * xhat).sum(0)}


def _kept_pass(s):
    q, scale = _rows8(s["X"])
    return q[:, :s["f"]].float() * scale.view(-1, 1)


def _act(kind, a):
    """The activation and its derivative."""
    if kind == NONE:
        return a, torch.ones_like(a)
    if kind == RELU:
        return a.clamp(min=0.0), (a > 0).float()
    if kind == ELU:
        return torch.where(a > 0, a, torch.expm1(a)), torch.exp(a.clamp(max=0.0))
    if kind == GELU:
        below = 0.5 * (1.0 + torch.erf(a * math.sqrt(0.5)))
        return a * below, below + a * torch.exp(-0.5 * a * a) * (1.0 / math.sqrt(2.0 * math.pi))
    g = 1.0 / (1.0 + torch.exp(-a))
    return (a * g, g * (1.0 + a * (1.0 - g))) if kind == SILU else (g, g * (1.0 - g))


def _linear_pass(s):
    z = s["X"] @ s["W"]
    if s["bias"]:
        z = z + s["b"]
    a, da = _act(s["act"], z)
    y = a + s["R"] if s["residual"] else a
    if not s["step"]:
        return y
    d = s["dY"] * da
    out = {"Y": y, "dW": s["X"].t() @ d, "dX": d @ s["W"].t()}
    return {**out, "db": d.sum(0)} if s["bias"] else out


def _back_pass(s):
    (xq, xs), (zq, zs) = s["X8"], s["Z8"]
    x = xq[:, :s["f_in"]].float() * xs.view(-1, 1) * s["gamma"]
    d = s["dY"] * _act(s["act"], zq[:, :s["f_out"]].float() * zs.view(-1, 1))[1]
    out = {"dW": x.t() @ d, "dX": d @ s["W"].t()}
    return {**out, "db": d.sum(0)} if s["bias"] else out


def _linear8_pass(s):
    (xq, xs), (wq, ws) = s["X8"], s["W8"]
    z = (xq.float() @ wq.float().t()) * xs.view(-1, 1) * ws       # the integers past the ends are zero
    y = _act(s["act"], z + s["b"] if s["bias"] else z)[0]
    return y + s["R"] if s["residual"] else y


# ---- the library's calls ---------------------------------------------------------------------------
def _kept_buffers(s, B):
    """Outputs and scratch that a program allocates once and keeps."""
    if "out" in s:
        return s["out"], s["ws"]
    new = functools.partial(torch.empty, dtype=torch.float32, device="cuda")
    n, kind, nbytes, out = s["n"], s["kind"], 0, {}

    def rows8(f):
        return B.Rows8(torch.empty(n, B.gnn_rows8_stride(f), dtype=torch.int8, device="cuda"), new(n))

    if kind == "kept":
        s["rows"], out = rows8(s["f"]), {"Y": new(n, s["f"])}
    elif kind == "rms":
        f = s["f"]
        out = {"Y": new(n, f)}
        s["rows"] = rows8(f) if s["keep"] else None
        if s["residual"]:
            out.update(H=new(n, f))
        if s["step"]:
            out.update(dR=new(n, f), dgamma=new(f))
            s["rstd"] = new(n)
            nbytes = B.gnn_rms_norm_workspace_bytes(n, f)
    else:
        m, k = s["f_in"], s["f_out"]
        s["act_id"] = getattr(B, "GNN_ACT_" + s["act"].upper())
        if kind == "linear8":
            s["X8"], s["W8"], out = B.Rows8(*s["X8"]), B.Rows8(*s["W8"]), {"Y": new(n, k)}
        else:
            back = kind == "back" or s["step"]
            nbytes = B.gnn_linear_workspace_bytes(back, n, m, k)
            if kind == "linear":
                out.update(Y=new(n, k))
                nbytes = max(nbytes, B.gnn_linear_workspace_bytes(False, n, m, k))
                s["Z"] = new(n, k) if s["keep"] and s["step"] else None
            else:
                s["X8"], s["Z8"] = B.Rows8(*s["X8"], columns=s["gamma"]), B.Rows8(*s["Z8"])
            if back:
                out.update(dW=new(m, k), dX=new(n, m))
                if s["bias"]:
                    out.update(db=new(k))
    s["out"], s["ws"] = out, B.alloc(nbytes)
    return s["out"], s["ws"]


def _own_pass(s):
    from paper_2308_12093_amd import binding as B

    o, ws = _kept_buffers(s, B)
    n, kind = s["n"], s["kind"]
    if kind == "kept":
        B.gnn_quantize_rows(n, s["f"], s["X"], None, s["rows"])
        B.gnn_dequantize_rows(n, s["f"], s["rows"], o["Y"])
        return o["Y"]
    if kind == "rms":
        f = s["f"]
        B.gnn_rms_norm_fwd(n, f, s["X"], s.get("R"), None, s["gamma"], EPS, o.get("H"), o["Y"], s["rows"], s.get("rstd"))
        if s["step"]:
            h = None if s["keep"] else o["H"] if s["residual"] else s["X"]
            B.gnn_rms_norm_bwd(n, f, h, s["rows"], s["rstd"], s["gamma"], None, s["dY"], s.get("dH"), o["dR"], None, o["dgamma"], ws)
        return o
    m, k, act = s["f_in"], s["f_out"], s["act_id"]
    if kind == "linear8":
        B.gnn_linear8_fwd(act, n, m, k, s["X8"], s["W8"], s["b"], s["R"], o["Y"])
        return o["Y"]
    if kind == "back":
        B.gnn_linear_bwd(act, n, m, k, None, s["X8"], s["W"], s["b"], None, s["Z8"], s["dY"], o["dW"], o.get("db"), o["dX"], ws)
        return o
    B.gnn_linear_fwd(act, n, m, k, s["X"], s["W"], s["b"], s["R"], o["Y"], s["Z"], ws)
    if not s["step"]:
        return o["Y"]
    B.gnn_linear_bwd(act, n, m, k, s["X"], None, s["W"], s["b"], s["Z"], None, s["dY"], o["dW"], o.get("db"), o["dX"], ws)
    return o


# ---- the definition in 64 bits -----------------------------------------------------------------------
def _held(x, factor=1.0):
    """The values that x stands for once it is in 8 bits.  The integers are defined by two operations rounded to floats."""
    largest = torch.linalg.vector_norm(x, ord=math.inf, dim=1, keepdim=True)
    largest = torch.where(largest == 0, torch.ones_like(largest), largest)
    per_unit = torch.full_like(largest, 127.0).div(largest).float().double()
    steps = (x * per_unit).float().double().round()
    return steps * (largest / 127.0) * factor


def _exact_act(kind, a):
    one = torch.ones_like(a)
    if kind == NONE:
        return a, one
    if kind == RELU:
        return a.relu(), (a > 0).double()
    if kind == ELU:
        slope = a.minimum(0.0 * one).exp()
        return a.relu() + torch.expm1(a.minimum(0.0 * one)), slope
    if kind == GELU:                                       # a times the normal distribution's integral up to a
        integral = torch.special.ndtr(a)
        return a * integral, integral + a * torch.exp(-a ** 2 / 2) / math.sqrt(2 * math.pi)
    up, down = torch.sigmoid(a), torch.sigmoid(-a)
    return (a * up, up + a * up * down) if kind == SILU else (up, up * down)


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    d = {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    if kind == "kept":
        return _held(d["X"])
    if kind == "rms":
        h = (s["X"] + s["R"]).double() if case["residual"] else d["X"]      # an array of floats, which the norm reads
        sigma = ((h ** 2).sum(1, keepdim=True) / case["f"] + EPS).sqrt()
        out = {"Y": d["gamma"] * h / sigma}
        if case["residual"]:
            out["H"] = d["X"] + d["R"]
        if not case["step"]:
            return out
        xhat = _held(h, 1.0 / sigma) if case["keep"] else h / sigma
        g = d["dY"] * d["gamma"]
        # the Jacobian of xhat: (1 - xhat xhat^T / f) / sigma
        dh = (g - xhat * (xhat * g).sum(1, keepdim=True) / case["f"]) / sigma
        return {**out, "dR": d.get("dH", 0.0) + dh, "dgamma": (d["dY"] * xhat).sum(0)}
    m, k = case["f_in"], case["f_out"]
    bias = d.get("b", torch.zeros(k, dtype=torch.float64, device="cuda"))
    if kind == "back":
        (xq, xs), (zq, zs) = s["X8"], s["Z8"]
        x = xq[:, :m].double() * xs.double()[:, None] * d["gamma"]
        slope = _exact_act(case["act"], zq[:, :k].double() * zs.double()[:, None])[1]
    elif kind == "linear8":
        (xq, xs), (wq, ws) = s["X8"], s["W8"]
        x, w = xq[:, :m].double() * xs.double()[:, None], wq[:, :m].double() * ws.double()[:, None]
        return _exact_act(case["act"], torch.addmm(bias, x, w.t()))[0] + d.get("R", 0.0)
    else:
        x = d["X"]
        a, slope = _exact_act(case["act"], torch.addmm(bias, x, d["W"]))
        y = a + d.get("R", 0.0)
        if not case["step"]:
            return y
    grad = d["dY"] * slope
    out = {"dW": torch.mm(x.t(), grad), "dX": torch.mm(grad, d["W"].t())}
    if kind == "linear":
        out["Y"] = y
    return {**out, "db": grad.sum(0)} if case["bias"] else out
