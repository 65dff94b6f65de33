"""The activations of the products, element by element, against their definitions: z goes through a product with one weight of 1.

In units of 2^-24 of the result.  Sigmoid: the argument of exp2 takes two roundings, worth 2 |z|; exp2 and the reciprocal are off by a
unit in the last place (2) each, 1 + e by 1; SiLU is rounded once more.  GELU below zero: exp(-z^2 / 2) takes three roundings in its
argument, worth 1.5 z^2, and exp2 2; t = 1 / (1 + 0.345 |z|) is off by 3, of which t Q(t) makes 2.4 times as much at most; the fit 1, the
polynomial's roundings 2, three products 3.  Above, 1 - Phi(-z) has half of that, of a result of one half at least, and 1."""
import numpy as np
import pytest
import torch
from scipy.special import expit, ndtr

from paper_2308_12093_amd import binding as B
from tests._util import dev, host

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.mark.parametrize("first,last", [(-87, -20), (-20, -8), (-8, -2), (-2, -0.5), (-0.5, 0), (0, 0.5), (0.5, 2), (2, 8), (8, 87)])
@pytest.mark.parametrize("act", ["sigmoid", "silu", "gelu"])
def test_off_by_no_more_than_stated(act, first, last):
    if act == "gelu":
        first = max(first, -12.9)
    if first >= last:
        pytest.skip("below the least normal float")
    n = 1 << 18
    z = np.linspace(first, last, n).astype(np.float32)
    Y = torch.full((n, 1), float("nan"), device="cuda")
    B.gnn_linear_fwd(getattr(B, "GNN_ACT_" + act.upper()), n, 1, 1, dev(z), torch.ones(1, device="cuda"), None, None, Y, None, B.alloc(256))
    got, x = host(Y)[:, 0].astype(np.float64), z.astype(np.float64)
    if act == "gelu":
        want, most = x * ndtr(x), np.where(x < 0, 16 + 1.5 * x * x, 17)
    else:
        want, most = expit(x) * (x if act == "silu" else 1.0), 6 + 2 * np.abs(x)
    assert (np.abs(got - want) <= most * U * np.abs(want) + 2.0 ** -149).all()
