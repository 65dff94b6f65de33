"""The gated feed-forward block against its definition in double precision.

Bounds in units of u = 2^-24.  The products take at most eight roundings per 16 indices and term, as the library's other products, so
[A | U] is within ez = (8 ceil(m / 16) + 8) u (|X||W| + |b|).  The activations have slopes of at most 1.13 and second derivatives of
at most 0.8 and are taken within 16 u of themselves (relative to max(1, |a|) for their slopes)."""
import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2308_12093_amd import binding as B
from tests._util import dev, host
from tests.test_gpu_norm import shifted, space, within

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
GATES = {"sigmoid": B.GNN_GATE_SIGMOID, "silu": B.GNN_GATE_SILU, "gelu": B.GNN_GATE_GELU}
NAN = float("nan")


class Case:
    def __init__(self, n, m, k, gate, bias=True, scale=1.0, seed=0):
        rng = np.random.default_rng(n + 7 * m + 31 * k + seed)
        f32 = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
        self.n, self.m, self.k, self.gate = n, m, k, gate
        self.X, self.W = f32(n, m) * np.float32(scale), f32(m, 2 * k) / np.float32(np.sqrt(m))
        self.b = f32(2 * k) / 4 if bias else None
        self.dH = f32(n, k)
        self.define()

    def define(self):
        k, gate = self.k, self.gate
        self.H, self.Z = blocks.gated_forward(self.X, self.W, self.b, gate)
        aX, aW = np.abs(self.X).astype(np.float64), np.abs(self.W).astype(np.float64)
        mag = aX @ aW + (0.0 if self.b is None else np.abs(self.b))
        ez = (8 * ((self.m + 15) // 16) + 8) * U * mag
        self.Z_most = ez
        a, u, ea, eu = self.Z[:, :k], self.Z[:, k:], ez[:, :k], ez[:, k:]
        g, dg = blocks.gate(gate, a)
        eg = 1.13 * ea + 16 * U * np.abs(g)
        edg = 0.8 * ea + 16 * U * np.maximum(1.0, np.abs(a))
        self.H_most = eg * np.abs(u) + (np.abs(g) + eg) * eu + 2 * U * np.abs(self.H)
        self.dW, self.db, self.dX, D = blocks.gated_backward(self.X, self.W, self.Z, self.dH, gate)
        d = np.abs(self.dH)
        eD = np.concatenate([d * (edg * np.abs(u) + (np.abs(dg) + edg) * eu), d * eg], 1) + 4 * U * np.abs(D)
        aD = np.abs(D) + eD
        self.dX_most = eD @ aW.T + (8 * ((2 * k + 15) // 16) + 8) * U * (aD @ aW.T)
        C = 64 + 8 * ((min(self.n, 4096) + 15) // 16)      # sums over the nodes: in float for 4096 of them at most, then in double
        self.dW_most = aX.T @ eD + C * U * (aX.T @ aD)
        self.db_most = eD.sum(0) + C * U * aD.sum(0)


def run(c, keep, by=0, want_dx=True):
    n, m, k = c.n, c.m, c.k
    X, W, dH, b = shifted(c.X, by), shifted(c.W, by), shifted(c.dH, by), None if c.b is None else shifted(c.b, by)
    H, Z, dW, db, dX = space(n, k, by), space(n, 2 * k, by), space(m, 2 * k, by), space(1, 2 * k, by), space(n, m, by)
    gate = GATES[c.gate]
    for back in (False, True):
        ws = B.alloc(B.gnn_gated_workspace_bytes(back, n, m, k))
        ws.fill_(255)
        if not back:
            B.gnn_gated_fwd(gate, n, m, k, X, W, b, H[0], Z[0] if keep else None, ws)
        else:
            B.gnn_gated_bwd(gate, n, m, k, X, W, b, Z[0] if keep else None, dH, dW[0], db[0], dX[0] if want_dx else None, ws)
    for _, end in (H, Z, dW, db, dX):
        assert bool((end == 7.0).all())
    return H[0], Z[0], dW[0], db[0][0], dX[0]


def check(c, got, keep):
    for t, name in zip(got, ("H", "Z", "dW", "db", "dX")):
        if name != "Z" or keep:
            within(t, getattr(c, name), getattr(c, name + "_most"), name)


SHAPES = [(1, 1, 1), (1, 256, 512), (2, 3, 5), (5, 16, 16), (7, 64, 33), (31, 100, 47), (33, 33, 65), (64, 512, 100), (129, 47, 130), (200, 5, 300),
          (300, 203, 259), (1000, 64, 64), (2049, 32, 96), (3001, 130, 70), (10000, 96, 48), (20011, 40, 129), (66001, 24, 36), (40000, 128, 256),
          (9000, 300, 515), (5000, 700, 33), (1, 2050, 7), (17, 1030, 1026),
          (3000, 40, 1200), (3000, 41, 1201), (40000, 20, 1), (40000, 3, 40), (30000, 300, 30), (40000, 301, 30), (33000, 50, 30), (40001, 33, 65),
          (2000, 512, 1000), (32767, 20, 40), (32768, 36, 130), (32767, 36, 130), (1, 520, 600), (33, 513, 514),
          (200, 260, 1025),
          (32767, 68, 130), (32768, 68, 130), (32769, 67, 129), (20011, 104, 129), (66001, 52, 68), (3000, 40, 2304), (3000, 41, 2401),
          (100000, 24, 65), (300000, 4, 20), (260000, 5, 30)]


@pytest.mark.parametrize("gate", ["sigmoid", "silu", "gelu"])
@pytest.mark.parametrize("n,m,k", SHAPES)
def test_gated_block(n, m, k, gate):
    big = n * (m + 2 * k) > 1 << 21
    c = Case(n, m, k, gate)
    for keep, by in ((True, 0), (False, 1)):
        check(c, run(c, keep, by), keep)
    if not big:
        c = Case(n, m, k, gate, bias=False)
        check(c, run(c, False, 0), False)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 31, 32, 33, 64, 65, 127, 128, 129, 255, 256, 257, 511, 513])
def test_few_rows(n):
    c = Case(n, 72, 40, "silu")
    for keep in (False, True):
        check(c, run(c, keep), keep)


@pytest.mark.parametrize("gate", ["sigmoid", "silu", "gelu"])
def test_far_from_zero(gate):
    """Gates that are shut or open all the way: exp and erf at their ends."""
    c = Case(400, 48, 50, gate, scale=60.0)
    assert np.abs(c.Z).max() > 100
    for keep in (False, True):
        check(c, run(c, keep), keep)


@pytest.mark.parametrize("n,m,k", [(4, 16, 16), (3000, 64, 64), (700, 130, 200)])
def test_without_an_input_gradient(n, m, k):
    c = Case(n, m, k, "gelu")
    got = run(c, True)
    again = run(c, True, want_dx=False)
    assert all(torch.equal(a, b) for a, b in zip(got[:4], again[:4])) and bool(torch.isnan(again[4]).all())


@pytest.mark.parametrize("n,m,k", [(3, 24, 20), (500, 64, 96), (5000, 64, 64), (20000, 64, 160), (3000, 40, 1200), (24000, 64, 200), (3000, 41, 2401)])
def test_what_is_not_finite_stays_where_it_belongs(n, m, k):
    """An infinite or NaN input spoils its row of H and dX, a NaN gradient the weights that it meets; every other row is exact."""
    c = Case(n, m, k, "silu")
    X = c.X.copy()
    X[1, 2], X[n - 1, 0] = np.inf, np.nan
    c.X, keep_X = X, c.X
    H, _, _, _, dX = (host(t) for t in run(c, False))
    c.X = keep_X
    rest = [i for i in range(n) if i not in (1, n - 1)]
    assert np.isnan(H[n - 1]).all() and not np.isfinite(H[1]).all()
    assert (np.abs(H[rest] - c.H[rest]) <= c.H_most[rest]).all()
    assert (np.abs(dX[rest] - c.dX[rest]) <= c.dX_most[rest]).all()
    dH = c.dH.copy()
    dH[0, 3] = np.nan
    c.dH, keep_dH = dH, c.dH
    dW, db = (host(t) for t in run(c, True)[2:4])
    c.dH = keep_dH
    cols = [j for j in range(2 * k) if j % k != 3]
    assert np.isnan(dW[:, [3, k + 3]]).all() and np.isnan(db[[3, k + 3]]).all()
    assert (np.abs(dW[:, cols] - c.dW[:, cols]) <= c.dW_most[:, cols]).all()


def test_an_infinite_product_is_infinite():
    """As with the fp32 instruction: parts of an infinity would make NaN of it."""
    for n, k in ((2, 32), (4000, 32), (40000, 160), (60000, 160)):
        c = Case(n, 32, k, "sigmoid", bias=False)
        W = np.abs(c.W)
        X = np.abs(c.X)
        X[0, 5] = np.inf
        c.X, c.W = X, W
        H = host(run(c, False)[0])
        assert np.isposinf(H[0]).all() and np.isfinite(H[1:]).all()


@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** 60])
def test_magnitudes_far_from_one(scale):
    for n, k in ((20, 40), (3000, 40), (20000, 160), (45000, 160)):
        c = Case(n, 40, k, "sigmoid", bias=False, scale=scale)
        H, _, dW, _, _ = run(c, False)
        within(H, c.H, c.H_most, "H")


@pytest.mark.parametrize("n,k", [(50, 48), (20000, 160), (45000, 160)])
def test_one_large_feature_beside_others(n, k):
    """A column of 1e8 whose weights are zero: the others keep their digits, in the products with the rows and with the columns."""
    c = Case(n, 40, k, "sigmoid", bias=False)
    c.X[:, 7], c.W[7] = 1e8, 0.0
    c.define()
    H, _, dW, _, dX = run(c, False)
    within(H, c.H, c.H_most, "H")
    within(dX, c.dX, c.dX_most, "dX")
    within(dW, c.dW, c.dW_most, "dW")


@pytest.mark.parametrize("n,k", [(50, 48), (20000, 160), (45000, 160)])
def test_rows_of_gradients_of_all_magnitudes(n, k):
    """dH of 1 down to 2^-60, and rows of zeros: every row of dX keeps its digits."""
    c = Case(n, 40, k, "silu")
    c.dH *= (2.0 ** -(np.arange(n) % 61)).astype(np.float32)[:, None]
    c.dH[::5] = 0.0
    c.define()
    for keep in (True, False):
        _, _, dW, db, dX = run(c, keep)
        within(dX, c.dX, c.dX_most, "dX")
        within(dW, c.dW, c.dW_most, "dW")
        within(db, c.db, c.db_most, "db")
    assert not host(dX)[::5].any()


def test_no_rows():
    dW, db = torch.full((4, 6), NAN, device="cuda"), torch.full((6,), NAN, device="cuda")
    ws = B.alloc(B.gnn_gated_workspace_bytes(True, 0, 4, 3))
    B.gnn_gated_bwd(0, 0, 4, 3, None, None, None, None, None, dW, db, None, ws)
    assert not dW.any() and not db.any()


@pytest.mark.parametrize("n,m,k", [(300, 64, 96), (5000, 64, 64), (1, 100, 60), (20000, 64, 160), (3000, 40, 1200), (24000, 64, 200),
                                   (3000, 40, 2304)])
def test_a_captured_step_replays(n, m, k):
    c = Case(n, m, k, "silu")
    X, W, b, dH = dev(c.X), dev(c.W), dev(c.b), dev(c.dH)
    out = dict(H=torch.empty(n, k, device="cuda"), Z=torch.empty(n, 2 * k, device="cuda"), dW=torch.empty(m, 2 * k, device="cuda"),
               db=torch.empty(2 * k, device="cuda"), dX=torch.empty(n, m, device="cuda"))
    ws = B.alloc(max(B.gnn_gated_workspace_bytes(back, n, m, k) for back in (0, 1)))

    def step(dW=out["dW"]):
        B.gnn_gated_fwd(1, n, m, k, X, W, b, out["H"], out["Z"], ws)
        B.gnn_gated_bwd(1, n, m, k, X, W, b, out["Z"], dH, dW, out["db"], out["dX"], ws)

    step()
    want = {name: t.clone() for name, t in out.items()}
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for _ in range(3):
        for t in out.values():
            t.fill_(NAN)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[name], want[name]) for name in out)
        step(torch.empty_like(out["dW"]))                  # eager, on the same workspace


def test_arrays_of_more_than_two_to_the_32_bytes():
    """[A | U] and D of 5 GB: the last rows of H and dX, and the weights' gradient, which every row is in."""
    n, m, k = (1 << 20) + 5, 16, 600
    gen = torch.Generator(device="cuda").manual_seed(2)
    X, W, dH = (torch.randn(*s, generator=gen, device="cuda") for s in ((n, m), (m, 2 * k), (n, k)))
    W /= 4.0
    H, Z, dX = torch.empty(n, k, device="cuda"), torch.empty(n, 2 * k, device="cuda"), torch.empty(n, m, device="cuda")
    dW, ws = torch.empty(m, 2 * k, device="cuda"), B.alloc(max(B.gnn_gated_workspace_bytes(back, n, m, k) for back in (0, 1)))
    for keep in (True, False):
        B.gnn_gated_fwd(GATES["sigmoid"], n, m, k, X, W, None, H, Z if keep else None, ws)
        B.gnn_gated_bwd(GATES["sigmoid"], n, m, k, X, W, None, Z if keep else None, dH, dW, None, dX, ws)
        tail = slice(n - 37, n)
        Wh, Xh, dHh = host(W), host(X[tail]), host(dH[tail])
        want, z = blocks.gated_forward(Xh, Wh, None, "sigmoid")
        _, _, want_dX, _ = blocks.gated_backward(Xh, Wh, z, dHh, "sigmoid")
        assert np.abs(host(H[tail]) - want).max() < 1e-5 and np.abs(host(dX[tail]) - want_dX).max() < 1e-3
        ref = torch.zeros(m, 2 * k, dtype=torch.float64, device="cuda")
        mag = torch.zeros_like(ref)
        for first in range(0, n, 1 << 17):
            x = X[first:first + (1 << 17)].double()
            zz = x @ W.double()
            s = torch.sigmoid(zz[:, :k])
            d = dH[first:first + (1 << 17)].double()
            D = torch.cat([d * zz[:, k:] * s * (1 - s), d * s], 1)
            ref += x.t() @ D
            mag += x.abs().t() @ D.abs()
        # of each term: the bound of the products (16 indices) and the gate's, and the sums of 4096 rows in float
        assert bool(((dW.double() - ref).abs() <= (2112 + 64) * U * mag).all())


@pytest.mark.parametrize("m", [4, 5, 7, 8, 16, 24, 31])
def test_short_reductions_are_those_of_floats(m):
    """One-hot rows, the commonest input of a layer on a graph: below 32 features a row of [A | U] is a row of W, bit for bit, few rows
    and many, kept or formed again (D, and with it dX, is the same then)."""
    for n, k in ((300, 40), (70000, 160), (33000, 515)):
        c = Case(n, m, k, "sigmoid", bias=False)
        which = np.arange(n) % m
        c.X[:] = 0.0
        c.X[np.arange(n), which] = 1.0
        c.define()
        kept = run(c, True)
        assert np.array_equal(host(kept[1]), c.W[which])
        check(c, kept, True)
        formed = run(c, False)
        check(c, formed, False)
        assert torch.equal(kept[0], formed[0])


@pytest.mark.parametrize("k", [2, 3, 5, 8, 12, 15])
def test_short_reductions_of_the_input_gradient(k):
    """D = [dH / 4 | dH / 2] exactly (a = 0, U = 1, sigmoid), so dX is one product of 2 k indices: its root mean square error is at most
    that of a chain of float multiplications and additions, within the scatter of 10^7 results (below 1 %, taken as 5)."""
    n, m = 40000, 260
    rng = np.random.default_rng(k)
    f32 = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
    X, W, dH = f32(n, m), f32(m, 2 * k), f32(n, k)
    Z = np.concatenate([np.zeros((n, k), np.float32), np.ones((n, k), np.float32)], 1)
    D = np.concatenate([dH / 4, dH / 2], 1)
    dX, dW = torch.empty(n, m, device="cuda"), torch.empty(m, 2 * k, device="cuda")
    ws = B.alloc(B.gnn_gated_workspace_bytes(True, n, m, k))
    B.gnn_gated_bwd(GATES["sigmoid"], n, m, k, dev(X), dev(W), None, dev(Z), dev(dH), dW, None, dX, ws)
    exact = D.astype(np.float64) @ W.astype(np.float64).T
    chain = np.zeros((n, m), np.float32)
    for j in range(2 * k):
        chain = (chain + np.outer(D[:, j].astype(np.float64), W[:, j])).astype(np.float32)
    rms = lambda a: np.sqrt(np.mean((a - exact) ** 2))  # noqa: E731
    assert rms(host(dX).astype(np.float64)) <= 1.05 * rms(chain)


@pytest.mark.parametrize("m,k", [(520, 600), (513, 514), (256, 1030), (700, 377), (16384, 500)])
def test_weights_of_one_row_have_the_products_of_floats(m, k):
    """One row: dW is x_i d_j, rounded once, with D as db has it (a sum of one)."""
    c = Case(1, m, k, "silu")
    for keep, by in ((True, 0), (False, 1)):
        got = run(c, keep, by)
        check(c, got, keep)
        assert torch.equal(got[2], dev(c.X).t() * got[3])


@pytest.mark.parametrize("n", [1, 2, 7, 15, 16, 31, 32, 33])
def test_weights_of_few_rows(n):
    """Wide weights, and [A | U] and D by the products of many rows as well (16384 x 500): dW within the error of a chain of n float
    multiplications and additions below 32 rows."""
    for m, k in ((512, 600), (513, 515), (16384, 500)):
        rng = np.random.default_rng(n)
        f32 = lambda *s: rng.standard_normal(s).astype(np.float32)  # noqa: E731
        X, W, dH = f32(n, m), f32(m, 2 * k), f32(n, k)
        Z = np.concatenate([np.zeros((n, k), np.float32), np.ones((n, k), np.float32)], 1)
        D = np.concatenate([dH / 4, dH / 2], 1)             # exactly: a = 0, U = 1, sigmoid
        dW, end = space(m, 2 * k)
        db, end2 = space(1, 2 * k)
        dX = torch.empty(n, m, device="cuda")
        ws = B.alloc(B.gnn_gated_workspace_bytes(True, n, m, k))
        ws.fill_(255)
        B.gnn_gated_bwd(GATES["sigmoid"], n, m, k, dev(X), dev(W), None, dev(Z), dev(dH), dW, db[0], dX, ws)
        assert bool((end == 7.0).all()) and bool((end2 == 7.0).all())
        terms = n if n < 32 else 8 * ((n + 15) // 16) + 8   # as above from there on
        mag = np.abs(X).astype(np.float64).T @ np.abs(D)
        within(dW, X.astype(np.float64).T @ D, terms * U * mag, "dW")
        within(db[0], D.astype(np.float64).sum(0), terms * U * np.abs(D).sum(0), "db")
        within(dX, D.astype(np.float64) @ W.astype(np.float64).T,
               (8 * ((2 * k + 15) // 16) + 8) * U * (np.abs(D) @ np.abs(W).astype(np.float64).T), "dX")


def signs(rng, *shape):
    return rng.choice(np.array([-1.0, 1.0], np.float32), shape)


def twelve_bits(rng, *shape):
    """Odd whole numbers of 2049 .. 4095 and either sign: twelve bits, of which one fp16 number holds eleven, so that each has a second
    part.  Sums of 4096 of them times +-1 stay below 2^24, exact in float in any order."""
    return (2 * rng.integers(1024, 2048, shape) + 1).astype(np.float32) * signs(rng, *shape)


@pytest.mark.parametrize("n,m,k", [(33, 512, 600), (5000, 64, 64), (9000, 300, 515), (40000, 128, 256), (33000, 50, 30), (40001, 33, 65),
                                   (2000, 512, 1000), (66001, 52, 68), (3000, 41, 1201), (100000, 40, 30), (32769, 67, 129)])
def test_second_parts_of_the_rows_reach_every_sum(n, m, k):
    """[A | U] = X W of whole numbers, gate columns zero: bit for bit as kept, and as formed again by what D sums up to: sixteen rows
    to a column, other ones for each, so that the sums stay exact (below 2^22, in steps of 1 / 4)."""
    rng = np.random.default_rng(n + m)
    c = Case(n, m, k, "sigmoid", bias=False)
    c.X = twelve_bits(rng, n, m)
    c.W = np.concatenate([np.zeros((m, k), np.float32), signs(rng, m, k)], 1)
    c.dH = np.zeros((n, k), np.float32)
    c.dH[rng.integers(0, n, (16, k)), np.arange(k)] = 1.0
    c.dH *= signs(rng, n, k)
    U = c.X.astype(np.float64) @ c.W[:, k:].astype(np.float64)
    kept, formed = run(c, True), run(c, False)
    assert np.array_equal(host(kept[1]), np.concatenate([np.zeros((n, k)), U], 1))
    for got in (kept, formed):
        assert np.array_equal(host(got[0]), U / 2)
        D = np.concatenate([c.dH * U / 4, c.dH / 2.0], 1)
        assert np.abs(D).sum(0).max() < 2.0 ** 22
        assert np.array_equal(host(got[3]), D.sum(0))
        assert np.array_equal(host(got[4]), D[:, k:] @ c.W[:, k:].astype(np.float64).T)


SECOND_PARTS = [(32, 512, 600), (33, 512, 600), (96, 512, 515), (200, 512, 1000), (4096, 300, 515), (4097, 300, 515), (9000, 300, 515),
                (9001, 130, 1201), (40000, 128, 256), (33000, 50, 30), (220000, 40, 30), (66001, 52, 68), (3000, 40, 1200), (40000, 300, 30)]


@pytest.mark.parametrize("n,m,k", SECOND_PARTS)
@pytest.mark.parametrize("of_x", [True, False])
def test_second_parts_reach_every_sum_of_the_gradients(n, m, k, of_x):
    """dW = X^T D and dX = D W^T of whole numbers, D = [dH / 4 | dH / 2] by a kept Z of a = 0, U = 1: bit for bit, over chunks of
    any number of steps, whichever of the operands has the second parts."""
    rng = np.random.default_rng(n + m + k)
    X, dH = (twelve_bits(rng, n, m), signs(rng, n, k)) if of_x else (signs(rng, n, m), twelve_bits(rng, n, k))
    W = signs(rng, m, 2 * k)
    Z = torch.cat([torch.zeros(n, k, device="cuda"), torch.ones(n, k, device="cuda")], 1)
    dW, db, dX = space(m, 2 * k), space(1, 2 * k), space(n, m)
    ws = B.alloc(B.gnn_gated_workspace_bytes(True, n, m, k))
    ws.fill_(255)
    B.gnn_gated_bwd(GATES["sigmoid"], n, m, k, dev(X), dev(W), None, Z, dev(dH), dW[0], db[0], dX[0], ws)
    D = np.concatenate([dH / 4, dH / 2], 1).astype(np.float64)
    assert np.array_equal(host(dW[0]), X.astype(np.float64).T @ D)
    assert np.array_equal(host(db[0][0]), D.sum(0))
    assert np.array_equal(host(dX[0]), D @ W.astype(np.float64).T)
    for _, end in (dW, db, dX):
        assert bool((end == 7.0).all())


@pytest.mark.parametrize("scale", [2.0 ** -100, 2.0 ** 60])
@pytest.mark.parametrize("n,k", [(20, 40), (3000, 40), (20000, 160), (45000, 160)])
def test_gradients_of_magnitudes_far_from_one(n, k, scale):
    """As above for X alone; a product or sum below 2^-126 may be taken as zero, each of which is worth that much at most."""
    c = Case(n, 40, k, "sigmoid", bias=False, scale=scale)
    c.dW_most = c.dW_most + n * 2.0 ** -126
    c.db_most, c.dX_most = c.db_most + n * 2.0 ** -126, c.dX_most + 2 * k * 2.0 ** -126
    for keep in (False, True):
        check(c, run(c, keep), False)


@pytest.mark.parametrize("n,m,k", [(2, 40, 32), (300, 512, 515), (4000, 32, 32), (40000, 40, 160), (60000, 40, 160), (9000, 300, 515),
                                   (33000, 300, 12)])
def test_infinite_sums_of_gradients_are_infinite(n, m, k):
    """Positive operands, one infinity in X and one in dH: a row and two columns of dW, a row of dX and two sums are +inf, nothing is NaN
    and the rest keeps its bounds."""
    rng = np.random.default_rng(n)
    pos = lambda *s: (0.5 + rng.random(s)).astype(np.float32)  # noqa: E731
    X, W, dH = pos(n, m), pos(m, 2 * k), pos(n, k)
    exact_D = np.concatenate([dH / 4, dH / 2], 1).astype(np.float64)
    want_dW, want_db, want_dX = X.astype(np.float64).T @ exact_D, exact_D.sum(0), exact_D @ W.astype(np.float64).T
    terms = 64 + 8 * ((min(n, 4096) + 15) // 16)
    X[n // 2, 3] = np.inf
    dH[n - 1, 5] = np.inf
    Z = torch.cat([torch.zeros(n, k, device="cuda"), torch.ones(n, k, device="cuda")], 1)
    dW, db, dX = (torch.full(s, NAN, device="cuda") for s in ((m, 2 * k), (2 * k,), (n, m)))
    ws = B.alloc(B.gnn_gated_workspace_bytes(True, n, m, k))
    B.gnn_gated_bwd(GATES["sigmoid"], n, m, k, dev(X), dev(W), None, Z, dev(dH), dW, db, dX, ws)
    dW, db, dX = host(dW), host(db), host(dX)
    inf_dW = np.zeros((m, 2 * k), bool)
    inf_dW[3], inf_dW[:, [5, k + 5]] = True, True
    assert np.array_equal(np.isposinf(dW), inf_dW) and np.isfinite(dW[~inf_dW]).all()
    assert (np.abs(dW - want_dW) <= terms * U * want_dW)[~inf_dW].all()
    assert np.isposinf(db[[5, k + 5]]).all() and np.isposinf(dX[n - 1]).all()
    rest = np.delete(np.arange(2 * k), [5, k + 5])
    assert (np.abs(db - want_db) <= terms * U * want_db)[rest].all()
    assert (np.abs(dX - want_dX)[:-1] <= (8 * ((2 * k + 15) // 16) + 8) * U * want_dX[:-1]).all()


@pytest.mark.parametrize("n,k", [(50, 48), (3000, 700), (45000, 160)])
def test_elements_far_below_the_largest_are_held_to_a_part_of_it(n, k):
    """A feature, and below a row, of 2^40 that meets zeros: the others, of magnitude 1, are held to 2^-50 of it each.  Scaled by 2^-26 the
    large one is 2^14; the second part, times 2^11, is rounded to a multiple of 2^-24, off by 2^-25: 2^-25 2^-11 2^26 = 2^-10."""
    m, held = 40, 2.0 ** -10
    c = Case(n, m, k, "sigmoid", bias=False)
    c.X[:, 7], c.W[7] = 2.0 ** 40, 0.0
    c.define()
    _, Z, _, _, _ = run(c, True)
    within(Z, c.Z, c.Z_most + held * np.abs(c.W).sum(0), "Z")
    c = Case(n, m, k, "sigmoid", bias=False)
    c.X[n // 3], c.dH[n // 3] = 2.0 ** 40, 0.0
    Z = torch.cat([torch.zeros(n, k, device="cuda"), torch.ones(n, k, device="cuda")], 1)
    dW, ws = torch.full((m, 2 * k), NAN, device="cuda"), B.alloc(B.gnn_gated_workspace_bytes(True, n, m, k))
    B.gnn_gated_bwd(GATES["sigmoid"], n, m, k, dev(c.X), dev(c.W), None, Z, dev(c.dH), dW, None, None, ws)
    D, X = np.concatenate([c.dH / 4, c.dH / 2], 1).astype(np.float64), c.X.astype(np.float64)
    X[n // 3] = 0.0
    C = 64 + 8 * ((min(n, 4096) + 15) // 16)
    within(dW, X.T @ D, C * U * (np.abs(X).T @ np.abs(D)) + held * np.abs(D).sum(0), "dW")


@pytest.mark.parametrize("n,m,k", [(70000, 16, 160), (20, 512, 600), (40000, 260, 7), (33000, 31, 515)])
def test_a_captured_step_of_short_products_replays(n, m, k):
    test_a_captured_step_replays(n, m, k)


@pytest.mark.parametrize("n,m,k", [(70000, 16, 160), (1, 513, 514), (33000, 31, 515), (31, 512, 600)])
def test_short_products_pass_on_what_is_not_finite(n, m, k):
    """An infinite or NaN input spoils its row of H, a NaN gradient the weights that it meets; all else keeps its bounds."""
    c = Case(n, m, k, "silu")
    keep_X = c.X
    c.X = keep_X.copy()
    c.X[n - 1, 0] = np.nan
    H = host(run(c, False)[0])
    c.X = keep_X
    assert np.isnan(H[n - 1]).all() and (np.abs(H - c.H) <= c.H_most)[:n - 1].all()
    keep_dH = c.dH
    c.dH = keep_dH.copy()
    c.dH[0, 3] = np.nan
    dW, db = (host(t) for t in run(c, True)[2:4])
    c.dH = keep_dH
    rest = [j for j in range(2 * k) if j % k != 3]
    assert np.isnan(dW[:, [3, k + 3]]).all() and np.isnan(db[[3, k + 3]]).all()
    assert (np.abs(dW - c.dW) <= c.dW_most)[:, rest].all()
