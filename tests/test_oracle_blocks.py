"""Pins of the double-precision definitions in oracle/blocks.py: published test vectors of the generator, torch autograd in
float64, central differences."""
import numpy as np
import pytest
import torch

from oracle import blocks


# The vectors that the authors of Philox publish with it (ten rounds): counter, key, words
VECTORS = [
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
     (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
]


@pytest.mark.parametrize("counter,key,words", VECTORS)
def test_generator_matches_the_published_vectors(counter, key, words):
    assert tuple(int(w) for w in blocks.philox4x32(counter, key)) == words


def test_dropout_factor_is_a_function_of_every_part_of_the_counter():
    base = blocks.dropout_factor(64, 37, 0.5, 123456789012345, 7, 2)
    assert set(np.unique(base)) == {0.0, 2.0}
    np.testing.assert_array_equal(base[:9, :5], blocks.dropout_factor(9, 5, 0.5, 123456789012345, 7, 2))
    for other in ((123456789012345, 8, 2), (123456789012345, 7, 3), (123456789012345 + (1 << 40), 7, 2), (-1, 7, 2)):
        assert 0.4 < np.mean(base != blocks.dropout_factor(64, 37, 0.5, *other)) < 0.6
    for p in (0.1, 0.6, 0.999):
        kept = np.mean(blocks.dropout_factor(1000, 101, p, 5, 1) > 0)
        assert abs(kept - (1 - p)) < 5 * np.sqrt(p * (1 - p) / 101000)
    assert (blocks.dropout_factor(5, 3, 0.0, 5, 1) == 1.0).all()


def test_dropped_values_are_zero_whatever_they_were():
    factor = np.array([[0.0, 2.0, 0.0, 2.0]])
    with np.errstate(invalid="ignore"):
        np.testing.assert_array_equal(blocks.dropout([[np.inf, 1.0, np.nan, -3.0]], factor), [[0.0, 2.0, 0.0, -6.0]])


@pytest.mark.parametrize("act", ["none", "relu", "elu"])
@pytest.mark.parametrize("n,f", [(1, 1), (5, 2), (9, 33)])
def test_layer_norm_against_autograd(n, f, act):
    rng = np.random.default_rng(n + f)
    X, gamma, beta, dY = rng.normal(size=(n, f)), rng.normal(size=f), rng.normal(size=f), rng.normal(size=(n, f))
    factor = blocks.dropout_factor(n, f, 0.3, 1, 2, 3)
    x, g, b = (torch.tensor(a, requires_grad=True) for a in (X, gamma, beta))
    z = torch.nn.functional.layer_norm(x, (f,), g, b, 1e-5)
    y = {"none": lambda v: v, "relu": torch.relu, "elu": torch.nn.functional.elu}[act](z) * torch.tensor(factor)
    y.backward(torch.tensor(dY))
    Y, Z = blocks.layer_norm_forward(X, gamma, beta, 1e-5, act, factor)
    np.testing.assert_allclose(Z, z.detach().numpy(), rtol=1e-10, atol=1e-12)
    np.testing.assert_allclose(Y, y.detach().numpy(), rtol=1e-10, atol=1e-12)
    for got, want in zip(blocks.layer_norm_backward(X, gamma, beta, 1e-5, dY, act, factor), (x, g, b)):
        np.testing.assert_allclose(got, want.grad.numpy(), rtol=1e-8, atol=1e-9)


@pytest.mark.parametrize("kind", ["sigmoid", "silu", "gelu"])
def test_gated_block_against_autograd_and_differences(kind):
    rng = np.random.default_rng(4)
    n, m, k = 7, 5, 6
    X, W, b, dH = rng.normal(size=(n, m)), rng.normal(size=(m, 2 * k)), rng.normal(size=2 * k), rng.normal(size=(n, k))
    x, w, bb = (torch.tensor(a, requires_grad=True) for a in (X, W, b))
    z = x @ w + bb
    fn = {"sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[kind]
    h = fn(z[:, :k]) * z[:, k:]
    h.backward(torch.tensor(dH))
    H, Z = blocks.gated_forward(X, W, b, kind)
    np.testing.assert_allclose(H, h.detach().numpy(), rtol=1e-12, atol=1e-13)
    dW, db, dX, _ = blocks.gated_backward(X, W, Z, dH, kind)
    for got, want in ((dW, w), (db, bb), (dX, x)):
        np.testing.assert_allclose(got, want.grad.numpy(), rtol=1e-10, atol=1e-12)
    # directional differences of sum(dH * H)
    value = lambda X_, W_: float((dH * blocks.gated_forward(X_, W_, b, kind)[0]).sum())  # noqa: E731
    e, vx, vw = 1e-5, rng.normal(size=X.shape), rng.normal(size=W.shape)
    slope = (value(X + e * vx, W + e * vw) - value(X - e * vx, W - e * vw)) / (2 * e)
    assert slope == pytest.approx(float((dX * vx).sum() + (dW * vw).sum()), rel=1e-7)


def test_layer_norm_gradient_against_differences():
    rng = np.random.default_rng(6)
    X, gamma, beta, dY = rng.normal(size=(4, 11)), rng.normal(size=11), rng.normal(size=11), rng.normal(size=(4, 11))
    value = lambda X_, g_: float((dY * blocks.layer_norm_forward(X_, g_, beta, 1e-5, "elu")[0]).sum())  # noqa: E731
    dX, dgamma, _ = blocks.layer_norm_backward(X, gamma, beta, 1e-5, dY, "elu")
    e, vx, vg = 1e-5, rng.normal(size=X.shape), rng.normal(size=11)
    slope = (value(X + e * vx, gamma + e * vg) - value(X - e * vx, gamma - e * vg)) / (2 * e)
    assert slope == pytest.approx(float((dX * vx).sum() + (dgamma * vg).sum()), rel=1e-7)


def test_the_composed_block_against_autograd():
    """tests/block_case.py: attention written densely, everything else by torch, gradients by autograd."""
    import oracle
    from tests import block_case as BC
    n, heads, k, q = 60, 2, 4, 10
    rowptr, col, t = BC.inputs(n, 3, heads, k, q, seed=1)
    rp, c, _ = oracle.add_self_loops_degree(rowptr, col)
    r = BC.define(rp, c, t, heads, step=5)
    v = {name: torch.tensor(a.astype(np.float64), requires_grad=name != "T") for name, a in t.items()}
    f = heads * k
    m1, m2 = (torch.tensor(blocks.dropout_factor(n, f, BC.P_DROP, BC.SEED, 5, s)) for s in (0, 1))
    y1 = torch.nn.functional.layer_norm(v["X"], (f,), v["g1"], v["b1"], BC.EPS)
    M = (y1 @ v["Wa"]).view(n, heads, k)
    logits = torch.einsum("nhk,hk->nh", M, v["a_src"])[:, None] + torch.einsum("nhk,hk->nh", M, v["a_dst"])[None]
    stored = torch.zeros(n, n, dtype=torch.bool)
    stored[np.repeat(np.arange(n), np.diff(rp)), c] = True
    alpha = torch.nn.functional.leaky_relu(logits, BC.SLOPE).masked_fill(~stored[..., None], -np.inf).softmax(dim=1)
    A = torch.einsum("ijh,jhk->ihk", alpha, M).reshape(n, f) + v["ba"]
    H = v["X"] + m1 * A
    z = torch.nn.functional.layer_norm(H, (f,), v["g2"], v["b2"], BC.EPS) @ v["W"] + v["b"]
    O = H + m2 * ((torch.nn.functional.silu(z[:, :q]) * z[:, q:]) @ v["Wd"])
    loss = 0.5 * ((O - v["T"]) ** 2).sum()
    loss.backward()
    assert r["loss"] == pytest.approx(loss.item(), rel=1e-12)
    np.testing.assert_allclose(r["O"], O.detach().numpy(), rtol=1e-10, atol=1e-11)
    names = dict(X="dX", g1="dg1", b1="db1", g2="dg2", b2="db2", Wa="dWa", a_src="da_src", a_dst="da_dst", ba="dba", W="dW", b="db", Wd="dWd")
    for name, grad in names.items():
        np.testing.assert_allclose(np.reshape(r[grad], v[name].shape), v[name].grad.numpy(), rtol=1e-8, atol=1e-9, err_msg=name)
