"""Refusals of rows in 8 bits, RMS norm and the products with their epilogue: every check comes before the first launch, so no GPU is
needed."""
import ctypes

import pytest

from paper_2308_12093_amd import binding as B

NULL, ONE, TWO = None, 256, 512                             # addresses that are never read
BAD, SMALL, NO = B.GNN_ERR_INVALID_ARG, B.GNN_ERR_BUFFER_TOO_SMALL, B.GNN_ERR_UNSUPPORTED


def rows(q=ONE, scale=ONE, columns=NULL):
    return ctypes.byref(B.gnn_rows8_t(q, scale, columns))


def drop(p=0.5, state=ONE):
    return ctypes.byref(B.gnn_dropout_t(p, 0, state))


ROWS = rows()
WRONG_ROWS = [rows(q=NULL), rows(scale=NULL), rows(q=264)]
WRONG_DROPS = [dict(p=-0.1), dict(p=1.0), dict(p=float("nan")), dict(p=2.0), dict(state=NULL), dict(state=260)]


def quantize(n=10, f=8, X=ONE, columns=NULL, out=ROWS):
    return B.lib.gnn_quantize_rows(n, f, X, columns, out, NULL)


def dequantize(n=10, f=8, out=ROWS, Y=ONE):
    return B.lib.gnn_dequantize_rows(n, f, out, Y, NULL)


def norm(n=10, f=8, X=ONE, R=NULL, d=NULL, eps=1e-5, H=NULL, Y=TWO, out=NULL):
    return B.lib.gnn_rms_norm_fwd(n, f, X, R, d, ONE, eps, H, Y, out, ONE, NULL)


def add_norm(R=ONE, H=ONE, **more):
    return norm(R=R, H=H, **more)


def back(n=10, f=8, H=ONE, out=NULL, rstd=ONE, d=NULL, dY=ONE, dH=NULL, dR=ONE, dX=TWO, dgamma=ONE, ws=ONE, nbytes=None):
    nbytes = B.gnn_rms_norm_workspace_bytes(n, f) if nbytes is None else nbytes
    return B.lib.gnn_rms_norm_bwd(n, f, H, out, rstd, ONE, d, dY, dH, dR, dX, dgamma, ws, nbytes, NULL)


def linear(act=0, n=10, m=8, k=4, X=ONE, W=ONE, R=NULL, Y=TWO, Z=NULL, ws=ONE, nbytes=None):
    nbytes = B.gnn_linear_workspace_bytes(False, n, m, k) if nbytes is None else nbytes
    return B.lib.gnn_linear_fwd(act, n, m, k, X, W, NULL, R, Y, Z, ws, nbytes, NULL)


def linear_back(act=0, n=10, m=8, k=4, X=ONE, X8=NULL, W=ONE, Z=NULL, Z8=NULL, dY=ONE, dW=ONE, dX=TWO, ws=ONE, nbytes=None):
    nbytes = B.gnn_linear_workspace_bytes(True, n, m, k) if nbytes is None else nbytes
    return B.lib.gnn_linear_bwd(act, n, m, k, X, X8, W, NULL, Z, Z8, dY, dW, NULL, dX, ws, nbytes, NULL)


def linear8(act=0, n=10, m=8, k=4, X=ROWS, W=ROWS, Y=TWO):
    return B.lib.gnn_linear8_fwd(act, n, m, k, X, W, NULL, NULL, Y, NULL)


@pytest.mark.parametrize("call", [quantize, dequantize, norm, add_norm, back])
def test_sizes_that_are_refused(call):
    more = dict(nbytes=1 << 62) if call is back else {}
    for wrong in (dict(n=-1), dict(f=0), dict(f=-4)):
        assert call(**wrong) == BAD, wrong
    for n, f in ((1, (1 << 24) + 1), (1, (1 << 31) - 1), (1 << 24, 4097)):
        assert call(n=n, f=f, **more) == NO, (n, f)


@pytest.mark.parametrize("call", [norm, add_norm, back])
def test_dropouts_that_are_refused(call):
    for wrong in WRONG_DROPS:
        assert call(d=drop(**wrong)) == BAD, wrong


def test_a_norm_alone_drops_nothing():
    assert norm(d=drop()) == BAD
    assert norm(H=ONE) == BAD


@pytest.mark.parametrize("call,needed", [(quantize, ["X", "out"]), (dequantize, ["out", "Y"]), (norm, ["X", "Y"]), (add_norm, ["X", "H", "Y"]),
                                         (back, ["H", "rstd", "dY", "ws"]), (linear, ["X", "W", "Y", "ws"]),
                                         (linear_back, ["X", "W", "dY", "dW", "ws"]), (linear8, ["X", "W", "Y"])])
def test_missing_arrays_are_refused(call, needed):
    for name in needed:
        assert call(**{name: NULL}) == BAD, name


@pytest.mark.parametrize("wrong", range(len(WRONG_ROWS)))
def test_rows_that_are_refused(wrong):
    w = WRONG_ROWS[wrong]
    for call, name in ((quantize, "out"), (dequantize, "out"), (norm, "out"), (add_norm, "out"), (linear8, "X"), (linear8, "W")):
        assert call(**{name: w}) == BAD, (call, name)
    assert back(H=NULL, out=w) == BAD
    assert linear_back(X=NULL, X8=w) == BAD
    assert linear_back(act=2, Z8=w) == BAD


def test_columns_where_they_are_not_read():
    c = rows(columns=ONE)
    for call, name in ((quantize, "out"), (norm, "out"), (add_norm, "out"), (linear8, "X"), (linear8, "W")):
        assert call(**{name: c}) == BAD, (call, name)


def test_one_source_of_each_input():
    assert back(H=ONE, out=ROWS) == BAD
    assert linear_back(X=ONE, X8=ROWS) == BAD
    assert linear_back(act=1, Z=ONE, Z8=ROWS) == BAD
    for act in range(1, 6):
        assert linear_back(act=act, X=NULL, X8=ROWS) == BAD


def test_arrays_that_must_differ():
    assert add_norm(H=ONE, Y=ONE) == BAD
    assert back(dR=ONE, dX=ONE) == BAD
    assert linear(Y=TWO, Z=TWO) == BAD


@pytest.mark.parametrize("call", [norm, add_norm])
def test_epsilons_that_are_refused(call):
    for eps in (0.0, -1e-5, 1e-40, float("nan"), float("inf")):
        assert call(eps=eps) == BAD, eps


@pytest.mark.parametrize("call", [linear, linear_back, linear8])
def test_products_that_are_refused(call):
    for wrong in (dict(act=-1), dict(act=6), dict(n=-1), dict(m=0), dict(k=0), dict(k=-2)):
        assert call(**wrong) == BAD, wrong
    more = {} if call is linear8 else dict(nbytes=1 << 60)
    assert call(k=1 << 30, **more) == NO
    if call is linear8:
        assert call(m=(1 << 17) + 1) == NO
        assert call(n=1 << 30, k=1 << 10) == NO
        return
    assert call(ws=260) == BAD
    assert call(nbytes=B.gnn_linear_workspace_bytes(call is linear_back, 10, 8, 4) - 1) == SMALL
    # 32 x 32 elements of Y a block: 256 x 65536; 32 rows and 64 columns of X: 8388608 x 2
    assert call(n=8176, m=3, k=1 << 21, nbytes=1 << 60) == NO
    assert call(n=1 << 28, m=65, k=64, nbytes=1 << 60) == NO


def test_the_last_sums_of_weights_that_no_grid_covers():
    assert linear_back(n=10, m=16384, k=32766, nbytes=1 << 60) == NO


def test_workspaces_that_are_refused():
    assert back(ws=260) == BAD
    assert back(nbytes=B.gnn_rms_norm_workspace_bytes(10, 8) - 1) == SMALL


def test_nothing_to_do_is_no_error():
    assert quantize(n=0, X=NULL, out=NULL) == B.GNN_OK
    assert dequantize(n=0, out=NULL, Y=NULL) == B.GNN_OK
    assert norm(n=0, X=NULL, Y=NULL) == B.GNN_OK
    assert back(n=0, H=NULL, rstd=NULL, dY=NULL, dR=NULL, dX=NULL, dgamma=NULL, ws=NULL, nbytes=0) == B.GNN_OK
    assert linear(n=0, X=NULL, W=NULL, Y=NULL, ws=NULL, nbytes=0) == B.GNN_OK
    assert linear8(n=0, X=NULL, W=NULL, Y=NULL) == B.GNN_OK


def test_strides_of_rows():
    assert [B.gnn_rows8_stride(f) for f in (1, 15, 16, 17, 203, 256)] == [16, 16, 16, 32, 208, 256]


@pytest.mark.parametrize("f", [1, 47, 256, 1000])
def test_a_workspace_for_the_most_rows_serves_fewer(f):
    rows_ = sorted({int(1.07 ** i) for i in range(300)} - {0} | {65535, 65536, 65537, 66000, 131072, 131073})
    rows_ = [n for n in rows_ if n < 1 << 24]
    sizes = [B.gnn_rms_norm_workspace_bytes(n, f) for n in rows_]
    assert sizes == sorted(sizes)
    for m in (1, 16, 100, 512):
        for back_ in (0, 1):
            sizes = [B.gnn_linear_workspace_bytes(back_, n, m, f) for n in rows_]
            assert sizes == sorted(sizes), (m, back_)


@pytest.mark.parametrize("m,k", [(512, 1024), (1024, 512), (512, 512), (300, 30), (128, 1024), (512, 7), (16, 512), (2048, 129), (3, 40)])
def test_a_workspace_serves_fewer_rows_on_both_sides_of_every_line(m, k):
    rows_ = sorted({n for p in range(23) for n in range(max(1, (1 << p) - 40), (1 << p) + 450)} | set(range(32700, 33300)))
    for back_ in (0, 1):
        sizes = [B.gnn_linear_workspace_bytes(back_, n, m, k) for n in rows_]
        fall = [(n, a, b) for n, a, b in zip(rows_[1:], sizes, sizes[1:]) if b < a]
        assert not fall, fall[:3]
