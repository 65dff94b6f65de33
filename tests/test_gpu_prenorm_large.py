"""The longest reductions of the product in 8 bits in its tiles of 128 x 128, and the sums over the rows of a norm of more than 2^32 bytes."""
import numpy as np
import pytest
import torch

from paper_2308_12093_amd import binding as B
from tests._util import dev, host
from tests.test_gpu_norm import EPS, NAN, U

pytestmark = pytest.mark.gpu


def integers(gen, rows, m):
    """[rows, m] of -127 .. 127, and something else behind the rows' ends."""
    room = torch.full((rows, B.gnn_rows8_stride(m)), 113, dtype=torch.int8, device="cuda")
    room[:, :m] = torch.randint(-127, 128, (rows, m), generator=gen, device="cuda", dtype=torch.int8)
    return room


@pytest.mark.parametrize("n,k", [(600, 600), (1000, 385)])
def test_largest_sums_in_tiles(n, k):
    """361 and 416 tiles of 32 x 32, where few rows end at 302: sums of +-127 x 127 x 2^17, the most that 32 bits have to hold."""
    m = 1 << 17
    gen = torch.Generator(device="cuda").manual_seed(n)
    sign = [torch.randint(0, 2, (r,), generator=gen, device="cuda", dtype=torch.int8) * 2 - 1 for r in (n, k)]
    X8, W8 = (B.Rows8((127 * s)[:, None].expand(-1, m).contiguous(), torch.ones(s.numel(), device="cuda")) for s in sign)
    Y = torch.full((n, k), NAN, device="cuda")
    B.gnn_linear8_fwd(B.GNN_ACT_NONE, n, m, k, X8, W8, None, None, Y)
    want = np.outer(host(sign[0]).astype(np.float64), host(sign[1]).astype(np.float64)) * (127.0 * 127.0 * m)
    assert np.array_equal(host(Y), want.astype(np.float32))


@pytest.mark.parametrize("m", [(1 << 17) - 1, (1 << 17) - 37, (1 << 17) - 64, 100_001])
def test_long_sums_in_tiles_that_end_inside_a_step(m):
    """Integers of every value, and others behind the rows' ends: each sum as the whole number that it is, rounded once."""
    n, k = 613, 607
    gen = torch.Generator(device="cuda").manual_seed(m)
    qx, qw = integers(gen, n, m), integers(gen, k, m)
    Y = torch.full((n, k), NAN, device="cuda")
    X8, W8 = B.Rows8(qx, torch.ones(n, device="cuda")), B.Rows8(qw, torch.ones(k, device="cuda"))
    B.gnn_linear8_fwd(B.GNN_ACT_NONE, n, m, k, X8, W8, None, None, Y)
    want = qx[:, :m].double() @ qw[:, :m].double().t().contiguous()        # whole numbers below 2^31: exact in double
    assert torch.equal(Y, want.float())


def test_dgamma_of_more_than_two_to_the_32_bytes():
    """Every row is in it: from H and from rows in 8 bits, against sums in double.  A group of lanes adds 256 rows at most in float, four
    groups and their blocks follow; an element of xhat takes up to three roundings."""
    n, f = 1_100_003, 1024
    gen = torch.Generator(device="cuda").manual_seed(6)
    X, dY = (torch.randn(n, f, generator=gen, device="cuda") for _ in range(2))
    X += 0.25
    gamma, rstd, rows = 1 + 0.1 * torch.randn(f, generator=gen, device="cuda"), torch.empty(n, device="cuda"), B.alloc_rows8(n, f)
    B.gnn_rms_norm_fwd(n, f, X, None, None, gamma, EPS, None, None, rows, rstd)
    dR, ws = torch.empty(n, f, device="cuda"), B.alloc(B.gnn_rms_norm_workspace_bytes(n, f))
    for held in (False, True):
        dg = torch.full((f,), NAN, device="cuda")
        ws.fill_(255)
        B.gnn_rms_norm_bwd(n, f, None if held else X, rows if held else None, rstd, gamma, None, dY, None, dR, None, dg, ws)
        want, most = (torch.zeros(f, dtype=torch.float64, device="cuda") for _ in range(2))
        for first in range(0, n, 1 << 17):
            part = slice(first, first + (1 << 17))
            d = dY[part].double() * (rows.q[part].double() * rows.scale[part].double()[:, None] if held
                                     else X[part].double() * rstd[part].double()[:, None])
            want += d.sum(0)
            most += d.abs().sum(0)
        assert bool(((dg.double() - want).abs() <= 303 * U * most).all())
        # rows at both ends and around 2^32 bytes
        at = torch.tensor([0, 1, n // 2, 1_048_575, 1_048_576, 1_048_577, n - 2, n - 1], device="cuda")
        xhat = (rows.q[at].double() * rows.scale[at].double()[:, None]) if held else X[at].double() * rstd[at].double()[:, None]
        g, r = dY[at].double() * gamma.double(), rstd[at].double()[:, None]
        grad = r * (g - xhat * (g * xhat).mean(1, keepdim=True))
        # the mean adds 16 products a lane and their sums over 64 lanes
        m = (g * xhat).abs().mean(1, keepdim=True)
        assert bool(((dR[at].double() - grad).abs() <= r * (8 * U * g.abs() + 40 * U * xhat.abs() * m)).all())
