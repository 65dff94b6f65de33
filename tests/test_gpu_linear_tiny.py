"""The products near the least normal float: rows and columns whose largest magnitudes are 2^-102 to 2^-130 lose no digits.

Operands are whole numbers of 19 bits times a power of two, few of them in a row or column and the others zero, and +-2^24.  Two fp16
numbers hold 22 bits and every sum of these stays below 2^24 units, so that the results are exact, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2308_12093_amd import binding as B
from tests._util import dev, host
from tests.test_gpu_linear import signs

pytestmark = pytest.mark.gpu

NAN = float("nan")
# pairs of 128 x 128 and of 128 x 256 outputs, ragged widths, chunks of rows that end inside a step; the last two by other kernels
SHAPES = [(33001, 132, 256), (70000, 260, 516), (33001, 131, 257), (16400, 516, 260), (40000, 128, 96), (300, 64, 96)]


def sparse(rng, shape, each, axis, exponent):
    """About `each` odd numbers of 19 bits along an axis, times 2^(exponent - 19): magnitudes of up to 2^exponent."""
    numbers = (2 * rng.integers(1 << 17, 1 << 18, shape) + 1) * rng.choice([-1, 1], shape)
    return (numbers * (rng.random(shape) < each / shape[axis])).astype(np.float32) * np.float32(2.0 ** (exponent - 19))


def exact(a, b, unit):
    want = a.astype(np.float64) @ b.astype(np.float64)
    assert (np.abs(a).astype(np.float64) @ np.abs(b).astype(np.float64)).max() < 2.0 ** 24 * unit
    return want


def product(X, W):
    (n, m), k = X.shape, W.shape[1]
    Y, ws = torch.full((n, k), NAN, device="cuda"), B.alloc(B.gnn_linear_workspace_bytes(False, n, m, k))
    B.gnn_linear_fwd(B.GNN_ACT_NONE, n, m, k, dev(X), dev(W), None, None, Y, None, ws)
    return host(Y)


def back(X, X8, W, dY):
    (m, k), n = W.shape, dY.shape[0]
    dW, dX = torch.full((m, k), NAN, device="cuda"), torch.full((n, m), NAN, device="cuda")
    ws = B.alloc(B.gnn_linear_workspace_bytes(True, n, m, k))
    B.gnn_linear_bwd(B.GNN_ACT_NONE, n, m, k, None if X is None else dev(X), X8, dev(W), None, None, None, dev(dY), dW, None, dX, ws)
    return host(dW), host(dX)


@pytest.mark.parametrize("exponent", [-102, -112, -118, -122, -125, -130])
@pytest.mark.parametrize("n,m,k", SHAPES)
def test_rows_and_columns_near_the_least_float(n, m, k, exponent):
    rng = np.random.default_rng(n - exponent)
    big, unit = np.float32(2.0 ** 24), 2.0 ** (exponent - 19 + 24)
    wide = lambda *s: signs(rng, *s) * big  # noqa: E731
    tiny = lambda shape, axis: sparse(rng, shape, 8, axis, exponent)  # noqa: E731
    X, W = tiny((n, m), 1), wide(m, k)                     # rows
    assert np.array_equal(product(X, W), exact(X, W, unit))
    X, W = wide(n, m), tiny((m, k), 0)                     # columns
    assert np.array_equal(product(X, W), exact(X, W, unit))
    X, W, dY = tiny((n, m), 0), wide(m, k), wide(n, k)     # columns of X
    assert np.array_equal(back(X, None, W, dY)[0], exact(X.T, dY, unit))
    X, dY = wide(n, m), tiny((n, k), 0)                    # columns of D, and its rows
    assert np.array_equal(back(X, None, W, dY)[0], exact(X.T, dY, unit))
    assert np.array_equal(back(X, None, W, dY)[1], exact(dY, W.T, unit))
    dY, W = wide(n, k), tiny((m, k), 1)                    # rows of W
    assert np.array_equal(back(X, None, W, dY)[1], exact(dY, W.T, unit))


@pytest.mark.parametrize("exponent", [-102, -112, -118, -122])
@pytest.mark.parametrize("n,m,k", SHAPES)
def test_rows_of_the_gradient_times_small_scales(n, m, k, exponent):
    """Integers of +-1 and a scale of 2^-60: D's rows times it are as small as above."""
    rng = np.random.default_rng(n - exponent)
    q = np.full((n, B.gnn_rows8_stride(m)), 33, np.int8)
    q[:, :m] = rng.choice([-1, 1], (n, m))
    dY, W = sparse(rng, (n, k), 8, 0, exponent + 60), signs(rng, m, k)
    X8 = B.Rows8(dev(q), torch.full((n,), 2.0 ** -60, device="cuda"))
    want = exact(q[:, :m].T * np.float32(2.0 ** -60), dY, 2.0 ** (exponent - 19))
    assert np.array_equal(back(None, X8, W, dY)[0], want)
