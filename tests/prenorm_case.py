"""A residual block that begins with an RMS norm, as the tests run it: inputs, and its definition in double precision.

    H = R + drop(X);  Y = gamma xhat(H);  A = act(Y W1 + b1);  O = A W2 + b2 + H;  loss = |O - T|^2 / 2

Backward is given the rows that were kept: xhat and Z = Y W1 + b1 and A, as they are or in 8 bits."""
import numpy as np

from oracle import blocks

EPS, P_DROP, SEED, ACT = 1e-5, 0.25, 91, "silu"


def inputs(n, f, q, seed):
    rng = np.random.default_rng(seed)
    f32 = lambda scale, *s: (rng.standard_normal(s) * scale).astype(np.float32)  # noqa: E731
    return dict(X=f32(1, n, f), R=f32(1, n, f), T=f32(1, n, f), gamma=1 + f32(0.1, f), W1=f32(f ** -0.5, f, q), b1=f32(0.1, q),
                W2=f32(q ** -0.5, q, f), b2=f32(0.1, f))


def forward(t, step):
    m = blocks.dropout_factor(*t["X"].shape, P_DROP, SEED, step)
    r = {"H": t["R"] + m * t["X"]}
    xhat, _ = blocks.rms_norm(r["H"], EPS)
    r["Y"] = xhat * t["gamma"]
    r["A"], r["Z"] = blocks.linear_forward(r["Y"], t["W1"], t["b1"], ACT)
    r["O"], _ = blocks.linear_forward(r["A"], t["W2"], t["b2"], "none", r["H"])
    return r


def backward(t, step, xhat, rstd, Z, A, dO):
    """The gradients, from what the kernels were given."""
    m = blocks.dropout_factor(*t["X"].shape, P_DROP, SEED, step)
    r = {}
    r["dW2"], r["db2"], r["dA"], _ = blocks.linear_backward(A, t["W2"], np.zeros_like(dO), dO, "none")
    r["dW1"], r["db1"], r["dY"], _ = blocks.linear_backward(xhat * t["gamma"], t["W1"], Z, r["dA"], ACT)
    dH, r["dgamma"] = blocks.rms_norm_backward(xhat, rstd, t["gamma"], r["dY"])
    r["dR"] = dO + dH
    r["dX"] = r["dR"] * m
    return r
