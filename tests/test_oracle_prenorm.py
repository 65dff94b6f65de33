"""The definitions of rows in 8 bits, RMS norm and the product with its epilogue, against autograd and against differences."""
import numpy as np
import pytest
import torch

from oracle import blocks

ACTS = {"none": lambda z: z, "relu": torch.relu, "elu": torch.nn.functional.elu, "sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu,
        "gelu": torch.nn.functional.gelu}


def test_rows_in_8_bits():
    rng = np.random.default_rng(1)
    X = (rng.standard_normal((40, 33)) * 10.0 ** rng.integers(-30, 30, (40, 1))).astype(np.float32)
    X[3] = 0.0
    X[5, 7] = np.inf
    X[6, 0] = np.nan
    X[7] = np.float32(1e-45) * np.arange(-16, 17)          # the least floats
    q, scale = blocks.held8(X)
    rest = [i for i in range(40) if i not in (5, 6)]
    assert np.isnan(scale[[5, 6]]).all() and not q[[5, 6, 3]].any() and scale[3] == 0.0
    held, x = q[rest] * scale[rest, None], X[rest].astype(np.float64)
    assert (np.abs(held - x) <= (0.5 + 127 * 2.0 ** -23) * scale[rest, None]).all()
    assert (np.abs(q[rest]).max(1) == np.where(scale[rest] > 0, 127, 0)).all()
    columns = rng.standard_normal(33).astype(np.float32)
    again, _ = blocks.held8(X[rest] * columns)
    assert np.array_equal(again, blocks.held8(X[rest], columns)[0])
    # ties go to the even neighbour
    assert blocks.held8(np.array([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5]]))[0].tolist() == [[127, 0, 2, 2, 0, -2]]


def test_rms_norm_against_autograd_and_differences():
    rng = np.random.default_rng(2)
    H, gamma, dY = rng.normal(size=(6, 11)), rng.normal(size=11), rng.normal(size=(6, 11))
    h, g = torch.tensor(H, requires_grad=True), torch.tensor(gamma, requires_grad=True)
    y = torch.nn.functional.rms_norm(h, (11,), g, 1e-5)
    y.backward(torch.tensor(dY))
    xhat, rstd = blocks.rms_norm(H, 1e-5)
    np.testing.assert_allclose(xhat * gamma, y.detach().numpy(), rtol=1e-12)
    dH, dgamma = blocks.rms_norm_backward(xhat, rstd, gamma, dY)
    np.testing.assert_allclose(dH, h.grad.numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(dgamma, g.grad.numpy(), rtol=1e-10, atol=1e-12)
    value = lambda H_, g_: float((dY * blocks.rms_norm(H_, 1e-5)[0] * g_).sum())  # noqa: E731
    e, vh, vg = 1e-5, rng.normal(size=H.shape), rng.normal(size=11)
    slope = (value(H + e * vh, gamma + e * vg) - value(H - e * vh, gamma - e * vg)) / (2 * e)
    assert slope == pytest.approx(float((dH * vh).sum() + (dgamma * vg).sum()), rel=1e-7)


@pytest.mark.parametrize("kind", list(ACTS))
def test_product_against_autograd_and_differences(kind):
    rng = np.random.default_rng(3)
    n, m, k = 7, 5, 6
    X, W, b, R, dY = rng.normal(size=(n, m)), rng.normal(size=(m, k)), rng.normal(size=k), rng.normal(size=(n, k)), rng.normal(size=(n, k))
    x, w, bb = (torch.tensor(a, requires_grad=True) for a in (X, W, b))
    y = ACTS[kind](x @ w + bb) + torch.tensor(R)
    y.backward(torch.tensor(dY))
    Y, Z = blocks.linear_forward(X, W, b, kind, R)
    np.testing.assert_allclose(Y, y.detach().numpy(), rtol=1e-12, atol=1e-13)
    dW, db, dX, _ = blocks.linear_backward(X, W, Z, dY, kind)
    for got, want in ((dW, w), (db, bb), (dX, x)):
        np.testing.assert_allclose(got, want.grad.numpy(), rtol=1e-10, atol=1e-12)
    value = lambda X_, W_: float((dY * blocks.linear_forward(X_, W_, b, kind, R)[0]).sum())  # noqa: E731
    e, vx, vw = 1e-6, rng.normal(size=X.shape), rng.normal(size=W.shape)
    slope = (value(X + e * vx, W + e * vw) - value(X - e * vx, W - e * vw)) / (2 * e)
    assert np.abs(Z).min() > 1e-4                          # no kink between
    assert slope == pytest.approx(float((dX * vx).sum() + (dW * vw).sum()), rel=1e-6)


@pytest.mark.parametrize("kept", [False, True])
def test_the_composed_block_against_autograd(kept):
    """tests/prenorm_case.py, gradients by autograd; what is kept in 8 bits is there an input of its own."""
    from tests import prenorm_case as PC
    n, f, q = 9, 12, 20
    t = PC.inputs(n, f, q, 5)
    r = PC.forward(t, 2)
    v = {name: torch.tensor(a.astype(np.float64), requires_grad=name != "T") for name, a in t.items()}
    m = torch.tensor(blocks.dropout_factor(n, f, PC.P_DROP, PC.SEED, 2))
    h = v["R"] + m * v["X"]
    rstd = 1 / torch.sqrt((h * h).mean(1, keepdim=True) + PC.EPS)
    z = (h * rstd * v["gamma"]) @ v["W1"] + v["b1"]
    a = torch.nn.functional.silu(z)
    o = a @ v["W2"] + v["b2"] + h
    np.testing.assert_allclose(r["O"], o.detach().numpy(), rtol=1e-12, atol=1e-12)
    if not kept:
        loss = 0.5 * ((o - v["T"]) ** 2).sum()
        loss.backward()
        xhat, s = blocks.rms_norm(r["H"], PC.EPS)
        g = PC.backward(t, 2, xhat, s, r["Z"], r["A"], r["O"] - t["T"])
        for name, grad in dict(X="dX", R="dR", gamma="dgamma", W1="dW1", b1="db1", W2="dW2", b2="db2").items():
            np.testing.assert_allclose(g[grad], v[name].grad.numpy(), rtol=1e-9, atol=1e-10, err_msg=name)
        return
    # 8 bits in place of xhat: the gradients differ by parts of a hundredth, not by a factor
    xhat, s = blocks.rms_norm(r["H"], PC.EPS)
    held = lambda x: (lambda q8, u: q8 * u[:, None])(*blocks.held8(x))  # noqa: E731
    plain = PC.backward(t, 2, xhat, s, r["Z"], r["A"], r["O"] - t["T"])
    g = PC.backward(t, 2, held(xhat), s, held(r["Z"]), held(r["A"]), r["O"] - t["T"])
    for name in plain:
        assert np.linalg.norm(g[name] - plain[name]) < 0.05 * np.linalg.norm(plain[name]), name
