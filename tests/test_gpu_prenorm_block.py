"""A residual block of RMS norm and two products as a network runs it, trained with its activations kept as they are and in 8 bits, eager and
captured, over three steps of the generator; and served in 8 bits."""
import numpy as np
import pytest
import torch

from oracle import blocks
from paper_2308_12093_amd import binding as B
from tests import prenorm_case as PC
from tests._util import assert_close, dev, host

pytestmark = pytest.mark.gpu

CASES = [(1, 16, 24, 0), (300, 48, 96, 1), (257, 33, 67, 2), (4000, 64, 130, 3), (33000, 128, 256, 4)]
ACT = B.GNN_ACT_SILU


class Block:
    def __init__(self, t, q, keep8):
        n, f = t["X"].shape
        self.n, self.f, self.q, self.keep8 = n, f, q, keep8
        self.d = {name: dev(a) for name, a in t.items()}
        e = lambda *s: torch.full(s, float("nan"), device="cuda")  # noqa: E731
        self.o = {name: e(n, f) for name in ("H", "Y", "O", "dO", "dY", "dR", "dX")}
        self.o.update({name: e(n, q) for name in ("Z", "A", "dA")}, rstd=e(n), loss=e(1), dW1=e(f, q), dW2=e(q, f), db1=e(q), db2=e(f), dgamma=e(f))
        self.rows = {name: B.alloc_rows8(n, w) for name, w in (("xhat", f), ("Z", q), ("A", q))}
        self.y8 = B.Rows8(self.rows["xhat"].q, self.rows["xhat"].scale, self.d["gamma"])
        sizes = [B.gnn_rms_norm_workspace_bytes(n, f), 4096]
        sizes += [B.gnn_linear_workspace_bytes(back, n, *s) for back in (0, 1) for s in ((f, q), (q, f))]
        self.ws = B.alloc(max(sizes))
        self.rng = torch.tensor([PC.SEED, 0], dtype=torch.int64, device="cuda")
        self.drop = B.Dropout(PC.P_DROP, self.rng, 0)

    def step(self):
        d, o, n, f, q, ws, rows = self.d, self.o, self.n, self.f, self.q, self.ws, self.rows
        keep = self.keep8
        B.gnn_rms_norm_fwd(n, f, d["X"], d["R"], self.drop, d["gamma"], PC.EPS, o["H"], o["Y"], rows["xhat"] if keep else None, o["rstd"])
        B.gnn_linear_fwd(ACT, n, f, q, o["Y"], d["W1"], d["b1"], None, o["A"], o["Z"], ws)
        if keep:
            B.gnn_quantize_rows(n, q, o["Z"], None, rows["Z"])
            B.gnn_quantize_rows(n, q, o["A"], None, rows["A"])
        B.gnn_linear_fwd(0, n, q, f, o["A"], d["W2"], d["b2"], o["H"], o["O"], None, ws)
        B.gnn_sum_squared_error(n * f, o["O"], d["T"], o["dO"], o["loss"], ws)
        one = lambda name, plain: (None, rows[name]) if keep else (plain, None)  # noqa: E731
        B.gnn_linear_bwd(0, n, q, f, *one("A", o["A"]), d["W2"], d["b2"], None, None, o["dO"], o["dW2"], o["db2"], o["dA"], ws)
        X, Z = ((None, self.y8), (None, rows["Z"])) if keep else ((o["Y"], None), (o["Z"], None))
        B.gnn_linear_bwd(ACT, n, f, q, *X, d["W1"], d["b1"], *Z, o["dA"], o["dW1"], o["db1"], o["dY"], ws)
        B.gnn_rms_norm_bwd(n, f, *one("xhat", o["H"]), o["rstd"], d["gamma"], self.drop, o["dY"], o["dO"], o["dR"], o["dX"], o["dgamma"], ws)
        B.gnn_rng_advance(self.rng)

    def held(self, name, width):
        rows = self.rows[name]
        return host(rows.q)[:, :width] * host(rows.scale).astype(np.float64)[:, None]


COMPARED = ("H", "Y", "Z", "A", "O", "dA", "dY", "dR", "dX", "dW1", "db1", "dW2", "db2", "dgamma")


@pytest.mark.parametrize("keep8", [False, True])
@pytest.mark.parametrize("n,f,q,seed", CASES)
def test_block(n, f, q, seed, keep8):
    t = PC.inputs(n, f, q, seed)
    block, eager = Block(t, q, keep8), []
    for step in range(3):
        block.step()
        r = PC.forward(t, step)
        o = {name: host(a).astype(np.float64) for name, a in block.o.items()}
        for name in ("H", "Y", "Z", "A", "O"):
            assert_close(o[name], r[name], f"step {step} {name}")
        rstd = o["rstd"][:, None]
        if keep8:
            # what 8 bits stand for is within half a step of a 127th of the row's largest magnitude
            for name, of in (("Z", "Z"), ("A", "A")):
                held = block.held(name, q)
                assert (np.abs(held - o[of]) <= (0.5 + 2e-5) * np.abs(o[of]).max(1, keepdims=True) / 127 + 1e-30).all()
            r.update(PC.backward(t, step, block.held("xhat", f), rstd, block.held("Z", q), block.held("A", q), o["dO"]))
        else:
            r.update(PC.backward(t, step, o["H"] * rstd, rstd, o["Z"], o["A"], o["dO"]))
        for name in ("dA", "dY", "dR", "dX"):
            assert_close(o[name], r[name], f"step {step} {name}")
        # sums over the rows: of magnitudes that grow with their root, each float off by 2^-24 of it
        for name in ("dW1", "db1", "dW2", "db2", "dgamma"):
            assert_close(o[name], r[name], f"step {step} {name}", tol=1e-4 * max(1.0, np.sqrt(n) / 50))
        eager.append({name: block.o[name].clone() for name in COMPARED})
    assert not torch.equal(eager[0]["H"], eager[1]["H"])
    block.rng[1] = 0
    torch.cuda.synchronize()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            block.step()
    for want in eager:
        for name in COMPARED:
            block.o[name].fill_(float("nan"))
        for rows in block.rows.values():
            rows.q.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        for name in COMPARED:
            assert torch.equal(block.o[name], want[name]), name


@pytest.mark.parametrize("n,f,q,seed", CASES)
def test_block_served_in_8_bits(n, f, q, seed):
    """gamma goes into the first weights; every product is that of the integers that it was given."""
    t = PC.inputs(n, f, q, seed)
    X8, A8 = B.alloc_rows8(n, f), B.alloc_rows8(n, q)
    W1, W2 = B.alloc_rows8(q, f), B.alloc_rows8(f, q)
    d = {name: dev(a) for name, a in t.items()}
    B.gnn_quantize_rows(q, f, d["W1"].t().contiguous(), d["gamma"], W1)
    B.gnn_quantize_rows(f, q, d["W2"].t().contiguous(), None, W2)
    H, A, O = (torch.full(s, float("nan"), device="cuda") for s in ((n, f), (n, q), (n, f)))
    B.gnn_rms_norm_fwd(n, f, d["X"], d["R"], None, None, PC.EPS, H, None, X8, None)
    B.gnn_linear8_fwd(ACT, n, f, q, X8, W1, d["b1"], None, A)
    B.gnn_quantize_rows(n, q, A, None, A8)
    B.gnn_linear8_fwd(0, n, q, f, A8, W2, d["b2"], H, O)
    value = lambda rows, w: host(rows.q)[:, :w] * host(rows.scale).astype(np.float64)[:, None]  # noqa: E731
    assert_close(host(H), t["R"].astype(np.float64) + t["X"], "H")
    a, _ = blocks.linear_forward(value(X8, f), value(W1, f).T, t["b1"], PC.ACT)
    assert_close(host(A), a, "A")
    o, _ = blocks.linear_forward(value(A8, q), value(W2, q).T, t["b2"], "none", host(H))
    assert_close(host(O), o, "O")
    # and the whole is the block, but for the 8 bits: each of the two products adds errors of a hundredth of its terms' root mean square
    whole = t["R"].astype(np.float64) + t["X"]
    y = blocks.rms_norm(whole, PC.EPS)[0] * t["gamma"]
    whole = blocks.linear_forward(blocks.linear_forward(y, t["W1"], t["b1"], PC.ACT)[0], t["W2"], t["b2"], "none", whole)[0]
    assert np.sqrt(((host(O) - whole) ** 2).mean()) < 0.05


def test_on_another_stream_than_the_current_ones_own():
    """Calls go to the current stream: work enqueued there before them is seen, and a captured step on it replays."""
    t = PC.inputs(500, 48, 96, 9)
    want = Block(t, 96, True)
    want.step()
    torch.cuda.synchronize()
    block, side = Block(t, 96, True), torch.cuda.Stream()
    x = block.d["X"].clone()
    block.d["X"].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        block.d["X"].copy_(x)
        block.step()
    torch.cuda.synchronize()
    for name in COMPARED:
        assert torch.equal(block.o[name], want.o[name]), name
