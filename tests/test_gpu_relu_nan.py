"""ReLU has no derivative at NaN: a NaN before it, which forward passes on, is in the gradients that meet it, as under ELU."""
import numpy as np
import pytest

from oracle import blocks
from tests._util import dev, host
from tests.test_gpu_linear import Case, backward, rows8
from tests.test_gpu_norm import Case as Norm
from tests.test_gpu_norm import EPS, run_norm

pytestmark = pytest.mark.gpu

# one launch; few rows; pairs in one scale; two scales; the fp32 instruction
SHAPES = [(5, 24, 20), (3000, 40, 60), (33001, 132, 256), (33001, 131, 257), (60000, 64, 50), (40000, 20, 200)]


def spoiled(t):
    return np.isnan(host(t))


@pytest.mark.parametrize("n,m,k", SHAPES)
def test_a_bias_that_is_nan(n, m, k):
    c = Case(n, m, k, "relu")
    c.b[3] = np.nan
    X, Z = dev(c.X), c.Z.astype(np.float32)
    Z[:, 3] = np.nan
    for how in (dict(), dict(Z=dev(Z))):
        dW, db, dX = backward(c, X, **how)
        for t in (dW, db.view(1, -1)):
            assert spoiled(t)[:, 3].all() and not np.delete(spoiled(t), 3, 1).any()
        assert spoiled(dX).all()                           # D is NaN in a column, which every row of dX meets


@pytest.mark.parametrize("n,m,k", SHAPES)
def test_a_row_lost_in_8_bits(n, m, k):
    c = Case(n, m, k, "relu")
    Z = c.Z.astype(np.float32)
    Z[n // 2, 1] = np.inf
    Z8, _ = rows8(Z)
    X8, _ = rows8(c.X)
    for x, x8 in ((dev(c.X), None), (None, X8)):
        dW, db, dX = backward(c, x, x8, None, Z8)
        assert spoiled(dW).all() and spoiled(db).all()
        assert spoiled(dX)[n // 2].all() and not np.delete(spoiled(dX), n // 2, 0).any()


@pytest.mark.parametrize("f", [6, 33, 96, 4100])
def test_layer_norm(f):
    c = Norm(9, f, "relu", 0.25)
    c.X[4, f // 2] = np.nan
    _, dX, dg, db = (host(t) for t in run_norm(c))
    want = blocks.layer_norm_backward(c.X, c.gamma, c.beta, EPS, c.dY, "relu", c.factor)
    for got, ref in zip((dX, dg, db), want):
        assert np.array_equal(np.isnan(got), np.isnan(ref))
    assert np.isnan(db).all() and np.isnan(dX).any(1).sum() == 1
