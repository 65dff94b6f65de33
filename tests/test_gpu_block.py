"""Layer norm, attention, dropout, residual connections and the gated feed-forward block together, as a network runs them: every
tensor and gradient against the definition in double precision, over three steps of the generator, eager and captured."""
import numpy as np
import pytest
import torch

import oracle
from oracle import blocks
from paper_2308_12093_amd import binding as B
from paper_2308_12093_amd import graphs
from tests import block_case as BC
from tests._util import assert_close, dev, host

pytestmark = pytest.mark.gpu

# (nodes, degree, heads, features a head, hidden of the feed-forward block, seed): few rows of the feed-forward block
CASES = [(300, 4, 3, 16, 40, 0), (257, 3, 2, 6, 33, 0), (5000, 2, 2, 16, 1024, 3)]


class Block:
    def __init__(self, g, heads, k, q, t, keep):
        n, f = t["X"].shape
        self.g, self.n, self.f, self.q = g, n, f, q
        self.d = {name: dev(a) for name, a in t.items()}
        self.plan = B.Plan(B.GNN_LAYER_GAT, n, g.nnz, f, k, heads=heads, has_bias=True, leaky_slope=BC.SLOPE)
        sizes = [self.plan.info.workspace_bytes, B.gnn_layer_norm_workspace_bytes(n, f), 4096,
                 *(B.gnn_gated_workspace_bytes(back, n, f, q) for back in (0, 1)),
                 *(B.gnn_gemm_workspace_bytes(ta, tb, *s) for ta, tb, s in ((0, 0, (n, f, q)), (0, 1, (n, q, f)), (1, 0, (q, f, n))))]
        self.ws, self.cache = B.alloc(max(sizes)), B.alloc(self.plan.info.cache_bytes)
        self.rng = torch.tensor([BC.SEED, 0], dtype=torch.int64, device="cuda")
        self.drop = [B.Dropout(BC.P_DROP, self.rng, site) for site in (0, 1)]
        e = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
        self.o = {name: e(n, f) for name in ("Y1", "A", "H", "Y2", "P", "O", "dO", "dP", "dY2", "dR", "dA", "dY1", "dXn", "dX")}
        self.o.update(G=e(n, q), dG=e(n, q), loss=e(1), dWd=e(q, f), dW=e(f, 2 * q), db=e(2 * q), dWa=e(f, f), da_src=e(heads, k),
                      da_dst=e(heads, k), dba=e(f), **{name: e(f) for name in ("dg1", "db1", "dg2", "db2")})
        self.stat = [e(n, 2) for _ in range(2)]
        self.Z = e(n, 2 * q) if keep else None

    def step(self):
        d, o, n, f, q, ws = self.d, self.o, self.n, self.f, self.q, self.ws
        B.gnn_layer_norm_fwd(n, f, d["X"], d["g1"], d["b1"], BC.EPS, B.GNN_ACT_NONE, None, o["Y1"], self.stat[0])
        B.gat_layer_fwd(self.plan, self.g, o["Y1"], d["Wa"], d["a_src"], d["a_dst"], d["ba"], o["A"], self.cache, ws)
        B.gnn_add_layer_norm_fwd(n, f, o["A"], d["X"], self.drop[0], d["g2"], d["b2"], BC.EPS, o["H"], o["Y2"], self.stat[1])
        B.gnn_gated_fwd(B.GNN_GATE_SILU, n, f, q, o["Y2"], d["W"], d["b"], o["G"], self.Z, ws)
        B.gnn_gemm(0, 0, n, f, q, o["G"], d["Wd"], o["P"], workspace=ws)
        B.gnn_dropout(n, f, o["P"], o["H"], self.drop[1], o["O"])
        B.gnn_sum_squared_error(n * f, o["O"], d["T"], o["dO"], o["loss"], ws)
        B.gnn_dropout(n, f, o["dO"], None, self.drop[1], o["dP"])
        B.gnn_gemm(1, 0, q, f, n, o["G"], o["dP"], o["dWd"], workspace=ws)
        B.gnn_gemm(0, 1, n, q, f, o["dP"], d["Wd"], o["dG"], workspace=ws)
        B.gnn_gated_bwd(B.GNN_GATE_SILU, n, f, q, o["Y2"], d["W"], d["b"], self.Z, o["dG"], o["dW"], o["db"], o["dY2"], ws)
        B.gnn_add_layer_norm_bwd(n, f, o["H"], self.stat[1], d["g2"], self.drop[0], o["dY2"], o["dO"], o["dR"], o["dA"], o["dg2"],
                                 o["db2"], ws)
        B.gat_layer_bwd(self.plan, self.g, o["Y1"], d["Wa"], d["a_src"], d["a_dst"], o["dA"], o["dWa"], o["da_src"], o["da_dst"],
                        o["dba"], o["dY1"], self.cache, ws)
        B.gnn_layer_norm_bwd(n, f, d["X"], self.stat[0], d["g1"], d["b1"], B.GNN_ACT_NONE, None, o["dY1"], o["dXn"], o["dg1"], o["db1"], ws)
        B.gnn_dropout(n, f, o["dXn"], o["dR"], None, o["dX"])
        B.gnn_rng_advance(self.rng)


COMPARED = ("Y1", "A", "H", "Y2", "G", "O", "dWd", "dW", "db", "dWa", "da_src", "da_dst", "dba", "dg1", "db1", "dg2", "db2", "dX")


@pytest.mark.parametrize("keep", [True, False])
@pytest.mark.parametrize("n,deg,heads,k,q,seed", CASES)
def test_block(n, deg, heads, k, q, seed, keep):
    rowptr, col, t = BC.inputs(n, deg, heads, k, q, seed)
    rp, c, _ = oracle.add_self_loops_degree(rowptr, col)
    block = Block(graphs.gat_graph(rowptr, col), heads, k, q, t, keep)
    eager = []
    for step in range(3):
        r = BC.define(rp, c, t, heads, step)
        assert r["nearest"] > 1e-5                          # no sign of LeakyReLU hangs on a rounding
        block.step()
        for name in COMPARED:
            assert_close(host(block.o[name]), np.reshape(r[name], block.o[name].shape), f"step {step} {name}")
        assert float(block.o["loss"]) == pytest.approx(r["loss"], rel=1e-5)
        eager.append({name: block.o[name].clone() for name in COMPARED})
    assert not torch.equal(eager[0]["O"], eager[1]["O"])
    block.rng[1] = 0
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            block.step()
    for want in eager:
        for name in COMPARED:
            block.o[name].fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        for name in COMPARED:
            assert torch.equal(block.o[name], want[name]), name


@pytest.mark.parametrize("keep", [True, False])
def test_block_of_many_rows(keep):
    """The feed-forward block's products on fp16 parts.  What is a row's own is compared with the whole block's definition.  A sum
    over 9000 rows adds up the roundings of all that stand before it (of magnitudes, sum |G| |dP|, of some thousands: 10^-4 each unit
    in the last place), so it is compared with its definition at the arrays that its kernel was given, within c u times the sum
    of magnitudes, u = 2^-24: c = 1 for the product of doubles' rounding to float, 2112 + 64 for the chunks of 4096 rows in float
    and the gate, 300 + 64 for the norm's and its statistics (off by 13 u of the row's mean magnitude: |xhat| + 1)."""
    n, deg, heads, k, q, seed = 9000, 2, 2, 16, 1024, 3
    rowptr, col, t = BC.inputs(n, deg, heads, k, q, seed)
    rp, c, _ = oracle.add_self_loops_degree(rowptr, col)
    block, u = Block(graphs.gat_graph(rowptr, col), heads, k, q, t, keep), 2.0 ** -24
    r = BC.define(rp, c, t, heads, 0)
    assert r["nearest"] > 1e-5
    block.step()
    o = {name: host(a).astype(np.float64) for name, a in block.o.items()}
    for name in ("Y1", "A", "H", "Y2", "G", "O", "dX"):
        assert_close(o[name], r[name], name)

    def within(name, ref, most):
        over = np.abs(o[name] - ref) - most
        assert over.max() <= 0, (name, over.max(), np.abs(o[name] - ref).max())

    ref = o["G"].T @ o["dP"]
    within("dWd", ref, u * (np.abs(ref) + 1e-6 * (np.abs(o["G"]).T @ np.abs(o["dP"]))))
    _, Z = blocks.gated_forward(o["Y2"], t["W"], t["b"], BC.GATE)
    dW, db, _, D = blocks.gated_backward(o["Y2"], t["W"], Z, o["dG"], BC.GATE)
    mag = np.abs(o["dG"]) * (1 + np.abs(Z[:, :q]) + np.abs(Z[:, q:])) * 2      # |D| and the gate's part in its error
    mag = np.concatenate([mag, mag], axis=1)
    within("dW", dW, (2112 + 64) * u * (np.abs(o["Y2"]).T @ mag))
    within("db", db, (2112 + 64) * u * mag.sum(axis=0))
    for X, dY, gamma, beta, dg, dbeta in ((o["H"], o["dY2"], "g2", "b2", "dg2", "db2"), (t["X"], o["dY1"], "g1", "b1", "dg1", "db1")):
        _, ref_g, ref_b = blocks.layer_norm_backward(X, t[gamma], t[beta], BC.EPS, dY)
        xhat = np.abs(blocks.normalise(X, BC.EPS)[0])
        within(dg, ref_g, 364 * u * (np.abs(dY) * (xhat + 1)).sum(axis=0))
        within(dbeta, ref_b, 364 * u * np.abs(dY).sum(axis=0))
