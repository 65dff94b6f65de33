"""Refusals of the operators between the layers: every check comes before the first launch, so no GPU is needed."""
import ctypes

import pytest

from paper_2308_12093_amd import binding as B

NULL, ONE, TWO = None, 256, 512                             # addresses that are never read
BAD, SMALL = B.GNN_ERR_INVALID_ARG, B.GNN_ERR_BUFFER_TOO_SMALL


def drop(p=0.5, state=ONE):
    return ctypes.byref(B.gnn_dropout_t(p, 0, state))


WRONG_DROPS = [dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(p=2.0), dict(state=NULL), dict(state=260)]


def dropout(n=10, f=8, X=ONE, R=NULL, d=NULL, Y=ONE):
    return B.lib.gnn_dropout(n, f, X, R, d, Y, NULL)


def forward(n=10, f=8, X=ONE, gamma=ONE, beta=ONE, eps=1e-5, act=0, d=NULL, Y=TWO, stat=ONE):
    return B.lib.gnn_layer_norm_fwd(n, f, X, gamma, beta, eps, act, d, Y, stat, NULL)


def backward(n=10, f=8, X=ONE, stat=ONE, act=0, d=NULL, dY=ONE, dX=TWO, dgamma=ONE, dbeta=ONE, ws=ONE, nbytes=None):
    nbytes = B.gnn_layer_norm_workspace_bytes(n, f) if nbytes is None else nbytes
    return B.lib.gnn_layer_norm_bwd(n, f, X, stat, ONE, ONE, act, d, dY, dX, dgamma, dbeta, ws, nbytes, NULL)


def add_forward(n=10, f=8, X=ONE, R=ONE, d=NULL, eps=1e-5, H=ONE, Y=TWO, stat=ONE):
    return B.lib.gnn_add_layer_norm_fwd(n, f, X, R, d, ONE, ONE, eps, H, Y, stat, NULL)


def add_backward(n=10, f=8, H=ONE, stat=ONE, d=NULL, dY=ONE, dH=ONE, dR=ONE, dX=TWO, dgamma=ONE, dbeta=ONE, ws=ONE, nbytes=None):
    nbytes = B.gnn_layer_norm_workspace_bytes(n, f) if nbytes is None else nbytes
    return B.lib.gnn_add_layer_norm_bwd(n, f, H, stat, ONE, d, dY, dH, dR, dX, dgamma, dbeta, ws, nbytes, NULL)


@pytest.mark.parametrize("call", [dropout, forward, backward, add_forward, add_backward])
def test_sizes_and_dropouts_that_are_refused(call):
    for wrong in (dict(n=-1), dict(f=0), dict(f=-4)):
        assert call(**wrong) == BAD, wrong
    for wrong in WRONG_DROPS:
        assert call(d=drop(**wrong)) == BAD, wrong


@pytest.mark.parametrize("call", [forward, backward, add_forward, add_backward])
def test_rows_that_no_grid_covers_are_refused(call):
    more = dict(nbytes=1 << 62) if call in (backward, add_backward) else {}
    for n, f in ((1, (1 << 24) + 1), (1, (1 << 31) - 1), (1 << 24, 4097)):
        assert call(n=n, f=f, **more) == B.GNN_ERR_UNSUPPORTED, (n, f)
    assert dropout(n=1, f=(1 << 30) + 1) == B.GNN_ERR_UNSUPPORTED


@pytest.mark.parametrize("call,needed", [(dropout, "XY"), (forward, ["X", "Y", "stat"]), (backward, ["X", "stat", "dY", "ws"]),
                                         (add_forward, ["X", "R", "H", "Y", "stat"]),
                                         (add_backward, ["H", "stat", "dY", "dR", "ws"])])
def test_missing_arrays_are_refused(call, needed):
    for name in needed:
        assert call(**{name: NULL}) == BAD, name


@pytest.mark.parametrize("call", [forward, add_forward])
def test_epsilons_that_are_refused(call):
    for eps in (0.0, -1e-5, 1e-40, float("nan"), float("inf")):
        assert call(eps=eps) == BAD, eps


@pytest.mark.parametrize("call", [forward, backward])
def test_activations_that_are_refused(call):
    for act in (-1, 3, 16):
        assert call(act=act) == BAD


@pytest.mark.parametrize("call", [backward, add_backward])
def test_workspaces_that_are_refused(call):
    assert call(ws=260) == BAD
    assert call(nbytes=B.gnn_layer_norm_workspace_bytes(10, 8) - 1) == SMALL


def test_arrays_that_must_differ():
    assert add_forward(H=ONE, Y=ONE) == BAD
    assert add_backward(dR=ONE, dX=ONE) == BAD


def test_nothing_to_do_is_no_error():
    assert dropout(n=0, X=NULL, Y=NULL) == B.GNN_OK
    assert forward(n=0, X=NULL, Y=NULL, stat=NULL) == B.GNN_OK
    assert add_forward(n=0, X=NULL, R=NULL, H=NULL, Y=NULL, stat=NULL) == B.GNN_OK
    assert backward(n=0, X=NULL, stat=NULL, dY=NULL, dX=NULL, dgamma=NULL, dbeta=NULL, ws=NULL, nbytes=0) == B.GNN_OK
    assert gated(n=0, X=NULL, W=NULL, H=NULL, ws=NULL, nbytes=0) == B.GNN_OK


def test_advancing_needs_an_aligned_state():
    assert B.lib.gnn_rng_advance(NULL, 1, NULL) == BAD
    assert B.lib.gnn_rng_advance(260, 1, NULL) == BAD


def gated(gate=0, n=10, m=8, k=4, X=ONE, W=ONE, H=TWO, ws=ONE, nbytes=None):
    nbytes = B.gnn_gated_workspace_bytes(False, n, m, k) if nbytes is None else nbytes
    return B.lib.gnn_gated_fwd(gate, n, m, k, X, W, NULL, H, NULL, ws, nbytes, NULL)


def gated_backward(gate=0, n=10, m=8, k=4, X=ONE, W=ONE, Z=NULL, dH=ONE, dW=ONE, dX=TWO, ws=ONE, nbytes=None):
    nbytes = B.gnn_gated_workspace_bytes(True, n, m, k) if nbytes is None else nbytes
    return B.lib.gnn_gated_bwd(gate, n, m, k, X, W, NULL, Z, dH, dW, NULL, dX, ws, nbytes, NULL)


@pytest.mark.parametrize("call,needed", [(gated, ["X", "W", "H", "ws"]), (gated_backward, ["X", "W", "dH", "dW", "ws"])])
def test_gated_blocks_that_are_refused(call, needed):
    for name in needed:
        assert call(**{name: NULL}) == BAD, name
    for wrong in (dict(gate=-1), dict(gate=3), dict(n=-1), dict(m=0), dict(k=0), dict(k=-2), dict(ws=260)):
        assert call(**wrong) == BAD, wrong
    assert call(nbytes=B.gnn_gated_workspace_bytes(call is gated_backward, 10, 8, 4) - 1) == SMALL
    assert call(k=1 << 30, nbytes=1 << 60) == B.GNN_ERR_UNSUPPORTED


@pytest.mark.parametrize("f", [1, 47, 256, 1000])
def test_a_workspace_for_the_most_rows_serves_fewer(f):
    rows = sorted({int(1.07 ** i) for i in range(300)} - {0} | {65535, 65536, 65537, 66000, 131072, 131073})
    rows = [n for n in rows if n < 1 << 24]
    sizes = [B.gnn_layer_norm_workspace_bytes(n, f) for n in rows]
    assert sizes == sorted(sizes)
    for m in (16, 100, 512):
        for back in (0, 1):
            sizes = [B.gnn_gated_workspace_bytes(back, n, m, f) for n in rows]
            assert sizes == sorted(sizes), (m, back)


@pytest.mark.parametrize("m,k", [(512, 1024), (1024, 512), (512, 512), (300, 30), (128, 1024), (512, 7), (16, 512), (2048, 129)])
def test_a_workspace_serves_fewer_rows_on_both_sides_of_every_line(m, k):
    """Row by row where blocks of rows change their size (32768) and around powers of two."""
    rows = sorted({n for p in range(23) for n in range(max(1, (1 << p) - 40), (1 << p) + 450)} | set(range(32700, 33300)))
    for back in (0, 1):
        sizes = [B.gnn_gated_workspace_bytes(back, n, m, k) for n in rows]
        fall = [(n, a, b) for n, a, b in zip(rows[1:], sizes, sizes[1:]) if b < a]
        assert not fall, fall[:3]


def test_gated_blocks_that_no_grid_covers_are_refused():
    """2^24 blocks of 256 threads and more: each of these is the sum or product of what one launch of the call would need."""
    no = B.GNN_ERR_UNSUPPORTED
    # the last sums of dW and of db together: 16384 x 32766 / 32 + 32766 / 32
    assert gated_backward(n=10, m=16384, k=16383, nbytes=1 << 60) == no
    # 32 x 32 elements of H a block: 256 x 65536
    for call in (gated, gated_backward):
        assert call(n=8176, m=3, k=1 << 21, nbytes=1 << 60) == no
    # 32 rows and 64 columns of X a block, 65 columns are two: 8388608 x 2
    for call in (gated, gated_backward):
        assert call(n=1 << 28, m=65, k=64, nbytes=1 << 60) == no
