"""Rows in 8 bits and the RMS norm against their definitions.

Bounds, in units of u = 2^-24 (half a step of a float).  Integers are those of the definition, bit for bit: it says how they are rounded.
A sum of f floats takes at most L = f / 64 + 12 roundings per term, all terms of a sum of squares have one sign, and so
  rstd        relative (L / 2 + 5) u                            =: r
  xhat        |xhat| (r + 2 u)                                  =: ex    (in 8 bits: of what the integers stand for)
  Y           |gamma| ex + u |Y|
The gradients follow by the same rules; a column's sum over the rows takes at most C = 300 roundings in float per term.
"""
import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2308_12093_amd import binding as B
from tests._util import dev, host
from tests.test_gpu_norm import EPS, NAN, SEED, SITE, STEP, U, shifted, space, state, within

pytestmark = pytest.mark.gpu


def room8(n, f):
    """Rows with a sentinel in everything that is not theirs."""
    rows = B.alloc_rows8(n + 1, f)
    rows.q.fill_(77)
    rows.scale.fill_(NAN)
    rows.scale[n:] = 7.0
    return rows


def unpack8(rows, n, f):
    """(integers, scale); what lies behind the last row is as it was, and the words behind a row's last."""
    q, scale = host(rows.q), host(rows.scale)
    assert (q[n:] == 77).all() and scale[n] == 7.0
    assert (q[:n, (f + 3) // 4 * 4:] == 77).all()
    return q[:n, :f], scale[:n]


class Case:
    def __init__(self, n, f, p=0.0, residual=True, scale=1.0, seed=0):
        rng = np.random.default_rng(1000 * n + f + seed)
        f32 = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
        self.n, self.f, self.p, self.residual = n, f, p, residual
        self.X = (f32(n, f) * np.float32(2.0) + np.float32(0.5)) * np.float32(scale)
        self.R = f32(n, f) * np.float32(scale) if residual else None
        self.gamma = 1 + f32(f) / 4
        self.dY, self.dH = f32(n, f), f32(n, f) if residual else None
        self.factor = blocks.dropout_factor(n, f, p, SEED, STEP, SITE)
        self.drop = B.Dropout(p, state(), SITE) if p else None


def forward(c, by=0, gamma=True, held=True, want_y=True):
    n, f = c.n, c.f
    X, R = shifted(c.X, by), shifted(c.R, by) if c.residual else None
    ga = shifted(c.gamma, by) if gamma else None
    H, Y, rstd = space(n, f, by), space(n, f, by), space(1, n)
    rows = room8(n, f) if held else None
    B.gnn_rms_norm_fwd(n, f, X, R, c.drop, ga, EPS, H[0] if c.residual else None, Y[0] if want_y else None, rows, rstd[0])
    for _, end in (H, Y, rstd):
        assert bool((end == 7.0).all())
    return H[0] if c.residual else X, Y[0], rows, rstd[0][0]


def check_forward(c, got, gamma=True):
    n, f, L = c.n, c.f, c.f / 64 + 12
    H, Y, rows, rstd = got
    h = host(H)
    if c.residual:
        scale = 1.0 / (1.0 - float(np.float32(c.p)))
        within(H, c.R.astype(np.float64) + blocks.dropout(c.X, c.factor), 3 * U * (np.abs(c.R) + scale * np.abs(c.X)), "H")
    xhat, exact = blocks.rms_norm(h, EPS)
    r = (L / 2 + 5) * U
    within(rstd.view(-1, 1), exact, r * exact, "rstd")
    g = c.gamma.astype(np.float64) if gamma else np.ones(f)
    if Y is not None:
        within(Y, g * xhat, (r + 3 * U) * np.abs(g * xhat), "Y")
    if rows is not None:
        q, s = unpack8(rows, n, f)
        want, unit = blocks.held8(h)
        assert np.array_equal(q, want)
        assert (np.abs(s - unit * exact[:, 0]) <= (r + 3 * U) * unit * exact[:, 0] + 2.0 ** -149).all()


def backward(c, H, rows, rstd, by=0, gamma=True, want_dx=True, want_dr=True, want_dg=True, over=None):
    n, f = c.n, c.f
    dY, dH, ga = shifted(c.dY, by), shifted(c.dH, by) if c.residual else None, shifted(c.gamma, by) if gamma else None
    dR, dX, dg = space(n, f, by), space(n, f, by), space(1, f, by)
    to = {"dY": dY, "dH": dH}.get(over, dR[0])
    ws = B.alloc(B.gnn_rms_norm_workspace_bytes(n, f))
    ws.fill_(255)                                          # NaN in float and in double
    B.gnn_rms_norm_bwd(n, f, H, rows, rstd, ga, c.drop, dY, dH, to if want_dr else None, dX[0] if want_dx else None,
                       dg[0] if want_dg else None, ws)
    for _, end in (dR, dX, dg):
        assert bool((end == 7.0).all())
    return to, dX[0], dg[0][0]


def check_backward(c, got, xhat, xhat_off, rstd, gamma=True):
    """xhat, rstd: what the pass was given; xhat_off: relative."""
    dR, dX, dg = got
    L = c.f / 64 + 12
    g = c.gamma.astype(np.float64) if gamma else np.ones(c.f)
    want, dgamma = blocks.rms_norm_backward(xhat, rstd, g, c.dY)
    ah, ag = np.abs(xhat), np.abs(c.dY * g)
    ex = (xhat_off + 2 * U) * ah
    m = np.abs((ag * ah).mean(1, keepdims=True))
    em = ((ag * ex).mean(1, keepdims=True) + (L + 4) * U * m)
    most = rstd * (3 * U * ag + ex * m + ah * em + 4 * U * (ag + ah * m)) + U * np.abs(want)
    if c.residual:
        want = want + c.dH
        most = most + U * np.abs(want)
    if dR is not None:
        within(dR, want, most, "dR")
    if dX is not None:
        within(dX, want * c.factor, c.factor * most + 2 * U * np.abs(want * c.factor), "dX")
        assert not host(dX)[c.factor == 0].any()
    if dg is not None:
        within(dg, dgamma, (np.abs(c.dY) * ex).sum(0) + 300 * U * np.abs(c.dY * xhat).sum(0), "dgamma")


def both_ways(c, by=0, gamma=True):
    H, Y, rows, rstd = got = forward(c, by, gamma)
    check_forward(c, got, gamma)
    r = host(rstd).astype(np.float64)[:, None]
    check_backward(c, backward(c, H, None, rstd, by, gamma), host(H) * r, U, r, gamma)
    q, s = unpack8(rows, c.n, c.f)
    check_backward(c, backward(c, None, rows, rstd, by, gamma), q * s.astype(np.float64)[:, None], U, r, gamma)


WIDTHS = [1, 2, 3, 4, 5, 7, 15, 16, 17, 31, 47, 64, 100, 128, 203, 256, 257, 512, 515, 1000, 1024, 1030, 2048, 2052, 4095, 4096, 4100, 8192, 20001]


@pytest.mark.parametrize("f", WIDTHS)
@pytest.mark.parametrize("n", [1, 2, 37])
def test_rms_norm(n, f):
    both_ways(Case(n, f))
    both_ways(Case(n, f, p=0.3))
    both_ways(Case(n, f, residual=False), by=1)
    both_ways(Case(n, f, residual=False), gamma=False)


@pytest.mark.parametrize("n,f", [(2708, 64), (3001, 203), (50000, 47), (9001, 1000), (40000, 512), (1025, 4100), (70001, 4), (300000, 3), (5000, 2050)])
def test_many_rows(n, f):
    for c, by in ((Case(n, f, p=0.1), 0), (Case(n, f, residual=False), 3)):
        both_ways(c, by)


@pytest.mark.parametrize("n,f", [(70000, 256), (20000, 1024), (5000, 4096), (140000, 128)])
def test_arrays_beyond_the_caches(n, f):
    """Read and written past the caches."""
    both_ways(Case(n, f, p=0.2))


@pytest.mark.parametrize("scale", [2.0 ** -75, 1e-20, 2.0 ** 40, 2.0 ** 54])
def test_magnitudes_far_from_one(scale):
    for f in (100, 5000):
        c = Case(20, f, scale=scale)
        got = forward(c)
        check_forward(c, got)


@pytest.mark.parametrize("f", [5, 64, 203, 4100])
def test_outputs_that_are_not_wanted_and_outputs_over_inputs(f):
    c = Case(33, f, p=0.3)
    H, Y, rows, rstd = forward(c)
    only = forward(c, want_y=False)
    assert bool(torch.isnan(only[1]).all()) and torch.equal(only[2].q, rows.q) and torch.equal(only[0], H)
    bare = forward(c, held=False)
    assert torch.equal(bare[1], Y) and torch.equal(bare[3], rstd)
    full = backward(c, H, None, rstd)
    for name in ("want_dx", "want_dr", "want_dg"):
        part = backward(c, H, None, rstd, **{name: False})
        for i, key in enumerate(("want_dr", "want_dx", "want_dg")):
            assert bool(torch.isnan(part[i]).all()) if key == name else torch.equal(part[i], full[i])
    for over in ("dY", "dH"):
        again = backward(c, H, None, rstd, over=over)
        assert all(torch.equal(a, b) for a, b in zip(again, full))
    # H over X, and over R; Y over X without a residual
    for which in (0, 1):
        a = [dev(c.X), dev(c.R)]
        Y2 = torch.empty_like(a[0])
        B.gnn_rms_norm_fwd(c.n, f, a[0], a[1], c.drop, dev(c.gamma), EPS, a[which], Y2, None, None)
        assert torch.equal(a[which], H) and torch.equal(Y2, Y)
    c = Case(33, f, residual=False)
    Y, X = forward(c)[1], dev(c.X)
    B.gnn_rms_norm_fwd(c.n, f, X, None, None, dev(c.gamma), EPS, None, X, None, None)
    assert torch.equal(X, Y)


@pytest.mark.parametrize("f", [1, 16, 47, 203, 1030, 4100])
def test_rows_of_zeros_and_rows_that_are_not_finite(f):
    c = Case(9, f, residual=False)
    c.X[2], c.X[4, f // 2], c.X[6, f - 1] = 0.0, np.inf, np.nan
    H, Y, rows, rstd = forward(c)
    Y, (q, s) = host(Y), unpack8(rows, 9, f)
    assert not Y[2].any() and not q[2].any() and s[2] == 0.0 and np.isfinite(host(rstd)[2])
    assert not np.isfinite(Y[4, f // 2]) and np.isnan(Y[6]).all()
    assert np.isnan(s[[4, 6]]).all() and not q[[4, 6]].any()
    rest = [0, 1, 3, 5, 7, 8]
    want, unit = blocks.held8(c.X[rest])
    assert np.array_equal(q[rest], want) and np.isfinite(Y[rest]).all() and np.isfinite(s[rest]).all()
    dR = host(backward(c, None, rows, rstd, want_dg=False)[0])
    assert np.isnan(dR[[4, 6]]).all() and np.isfinite(dR[rest + [2]]).all()


def test_squares_beyond_the_largest_float():
    c = Case(3, 40, residual=False)
    c.X[1] = 2.0 ** 64
    Y, rows = forward(c)[1:3]
    q, s = unpack8(rows, 3, 40)
    assert not host(Y)[1].any() and s[1] == 0.0 and np.isfinite(host(Y)).all()


@pytest.mark.parametrize("n,f", [(1, 1), (3, 5), (40, 16), (7, 203), (2708, 64), (40000, 131), (70000, 256), (9, 4097), (300, 6000)])
@pytest.mark.parametrize("columns", [False, True])
def test_rows_in_8_bits(n, f, columns):
    rng = np.random.default_rng(n + f)
    X = (rng.standard_normal((n, f)) * 10.0 ** rng.integers(-36, 30, (n, 1))).astype(np.float32)
    cols = rng.standard_normal(f).astype(np.float32) if columns else None
    for by in (0, 1):
        rows = room8(n, f)
        B.gnn_quantize_rows(n, f, shifted(X, by), None if cols is None else shifted(cols, by), rows)
        q, s = unpack8(rows, n, f)
        want, unit = blocks.held8(X, cols)
        assert np.array_equal(q, want)
        assert (np.abs(s - unit) <= U * unit + 2.0 ** -149).all()
        # read back, times columns
        back = B.Rows8(rows.q, rows.scale, None if cols is None else shifted(cols, by))
        Y = space(n, f, by)
        B.gnn_dequantize_rows(n, f, back, Y[0])
        held = q * s.astype(np.float64)[:, None] * (1.0 if cols is None else cols.astype(np.float64))
        within(Y[0], held, 2 * U * np.abs(held) + 2.0 ** -148 * (1.0 if cols is None else 1.0 + np.abs(cols)), "held")
        assert bool((Y[1] == 7.0).all())


def test_the_least_and_the_largest_floats_in_8_bits():
    top = float(np.finfo(np.float32).max)
    X = np.stack([np.float32(1e-45) * np.arange(-20, 20), np.linspace(-top, top, 40), np.full(40, 1.2e-38), np.linspace(-9e-31, 7e-31, 40),
                  np.linspace(0, 7.8886090522101e-31, 40)]).astype(np.float32)
    rows = room8(5, 40)
    B.gnn_quantize_rows(5, 40, dev(X), None, rows)
    q, s = unpack8(rows, 5, 40)
    want, unit = blocks.held8(X)
    assert np.array_equal(q, want) and (np.abs(s - unit) <= U * unit + 2.0 ** -149).all()


def test_no_rows():
    g = torch.full((7,), NAN, device="cuda")
    B.gnn_rms_norm_bwd(0, 7, None, None, None, None, None, None, None, None, None, g, B.alloc(B.gnn_rms_norm_workspace_bytes(0, 7)))
    assert not host(g).any()


@pytest.mark.parametrize("n,f", [(300, 47), (20000, 512), (70, 5000)])
def test_a_captured_step_replays(n, f):
    c = Case(n, f, p=0.25)
    X, R, ga, dY, dH = (dev(a) for a in (c.X, c.R, c.gamma, c.dY, c.dH))
    rng = state()
    drop = B.Dropout(0.25, rng, SITE)
    o = {k: torch.full((n, f), NAN, device="cuda") for k in ("H", "Y", "dR", "dX")}
    o.update(rstd=torch.full((n,), NAN, device="cuda"), dg=torch.full((f,), NAN, device="cuda"))
    rows, ws = B.alloc_rows8(n, f), B.alloc(B.gnn_rms_norm_workspace_bytes(n, f))

    def step():
        B.gnn_rms_norm_fwd(n, f, X, R, drop, ga, EPS, o["H"], o["Y"], rows, o["rstd"])
        B.gnn_rms_norm_bwd(n, f, None, rows, o["rstd"], ga, drop, dY, dH, o["dR"], o["dX"], o["dg"], ws)
        B.gnn_rng_advance(rng)

    eager = []
    for _ in range(3):
        step()
        eager.append({k: v.clone() for k, v in o.items()})
    assert not torch.equal(eager[0]["H"], eager[1]["H"])
    rng.copy_(state())
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for want in eager:
        for v in o.values():
            v.fill_(NAN)
        rows.q.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o[k], want[k]) for k in o)


def test_arrays_of_more_than_two_to_the_32_bytes():
    n, f = 1_100_003, 1024
    X = torch.randn(n, f, device="cuda")
    gamma, Y, rstd, rows = 1 + 0.1 * torch.randn(f, device="cuda"), torch.empty(n, f, device="cuda"), torch.empty(n, device="cuda"), B.alloc_rows8(n, f)
    B.gnn_rms_norm_fwd(n, f, X, None, None, gamma, EPS, None, Y, rows, rstd)
    at = torch.tensor([0, 1, n // 2, 1_048_575, 1_048_576, 1_048_577, n - 2, n - 1], device="cuda")
    want, unit = blocks.held8(host(X[at]))
    assert np.array_equal(host(rows.q[at]), want)
    xhat, exact = blocks.rms_norm(host(X[at]), EPS)
    assert np.allclose(host(Y[at]), xhat * host(gamma), rtol=1e-5, atol=1e-30)
    dR, dg, ws = Y, torch.empty(f, device="cuda"), B.alloc(B.gnn_rms_norm_workspace_bytes(n, f))
    dY = X
    B.gnn_rms_norm_bwd(n, f, None, rows, rstd, gamma, None, dY, None, dR, None, dg, ws)
    held = host(rows.q[at]) * host(rows.scale[at]).astype(np.float64)[:, None]
    grad, _ = blocks.rms_norm_backward(held, exact, host(gamma), host(dY[at]))
    assert np.allclose(host(dR[at]), grad, rtol=1e-4, atol=1e-4)
    back = Y
    B.gnn_dequantize_rows(n, f, rows, back)
    assert np.allclose(host(back[at]), held, rtol=1e-6)
