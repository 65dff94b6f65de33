"""``binding.Rows8``: what it refuses before a kernel could read or write outside of its tensors, and tensors put in others' place.  No
launch but where marked, so no GPU is needed."""
import copy

import numpy as np
import pytest
import torch

from paper_2308_12093_amd import binding as B

N, F = 12, 20                                               # rows of 32 bytes
INT8 = dict(dtype=torch.int8)


@pytest.fixture
def no_stream(monkeypatch):
    monkeypatch.setattr(B, "_stream", lambda: None)


def rows(n=N, f=F, columns=None):
    return B.Rows8(torch.zeros(n, B.gnn_rows8_stride(f), **INT8), torch.zeros(n), columns)


def refused(call, *args):
    with pytest.raises(B.GnnError) as e:
        call(*args)
    return e.value.status == B.GNN_ERR_INVALID_ARG


@pytest.mark.parametrize("q", [torch.zeros(N, 32, dtype=torch.uint8), torch.zeros(N, 32), None,
                               torch.zeros(32, N, **INT8).t(), torch.zeros(N, 64, **INT8)[:, :32], torch.zeros(2 * N, 32, **INT8)[::2]])
def test_integers_that_are_refused(q):
    assert refused(B.Rows8, q, torch.zeros(N))


@pytest.mark.parametrize("scale", [None, torch.zeros(N, dtype=torch.float64), torch.zeros(2 * N)[::2], torch.zeros(N, dtype=torch.float16)])
def test_scales_and_columns_that_are_refused(scale):
    q = torch.zeros(N, 32, **INT8)
    assert refused(B.Rows8, q, scale)
    if scale is not None:
        assert refused(B.Rows8, q, torch.zeros(N), scale)


def calls(X8):
    """Every call that takes [N, F] in 8 bits; those it writes and those it reads."""
    x, ws, W8 = torch.zeros(N, F), torch.zeros(1 << 20, dtype=torch.uint8), rows(7, F)
    y, g = torch.zeros(N, 7), torch.zeros(F)
    return [
        (B.gnn_quantize_rows, N, F, x, None, X8),
        (B.gnn_dequantize_rows, N, F, X8, x),
        (B.gnn_rms_norm_fwd, N, F, x, None, None, None, 1e-5, None, x, X8, g),
        (B.gnn_rms_norm_bwd, N, F, None, X8, g, None, None, x, None, x, None, None, ws),
        (B.gnn_linear_bwd, 0, N, F, 7, None, X8, x, None, None, None, y, x, None, None, ws),
        (B.gnn_linear_bwd, 1, N, 7, F, y, None, x, None, None, X8, x, x, None, None, ws),
        (B.gnn_linear8_fwd, 0, N, F, 7, X8, W8, None, None, y),
        (B.gnn_linear8_fwd, 0, 7, F, N, W8, X8, None, None, y),
    ]


@pytest.mark.parametrize("i", range(8))
def test_rows_too_few_and_strides_that_do_not_fit(i, no_stream):
    """An int8 [N, F] tensor, whose last row would be written past its end; a wider stride; rows or scales that end early."""
    for q, scale in (((N, F), N), ((N, 48), N), ((N, 16), N), ((N - 1, 32), N), (N * 32 - 1, N), ((N, 32), N - 1)):
        X8 = B.Rows8(torch.zeros(q, **INT8), torch.zeros(scale))
        call, *args = calls(X8)[i]
        assert refused(call, *args), (call.__name__, q, scale)


@pytest.mark.parametrize("i", [1, 4, 5])
def test_columns_too_few(i, no_stream):
    call, *args = calls(rows(columns=torch.zeros(F - 1)))[i]
    assert refused(call, *args)


def test_more_rows_and_columns_than_are_needed():
    flat = B.Rows8(torch.zeros((N + 3) * 32, **INT8), torch.zeros(N + 3))
    for room in (rows(N + 3, 30, torch.zeros(40)), flat):
        for n in (0, 1, N, N + 3):
            for f in (17, F, 30, 32):
                room._look(n, f)


def test_columns_given_later_are_the_columns(no_stream):
    """gnn_quantize_rows refuses columns in what it writes: as soon as they are there, and no longer."""
    room, x = rows(), torch.zeros(N, F)
    room.columns = torch.ones(F)
    assert refused(B.gnn_quantize_rows, N, F, x, None, room)
    room.columns = None
    assert not room.c.columns
    q, scale = torch.zeros(N, 32, **INT8), torch.zeros(N)
    room.q, room.scale = q, scale
    assert (room.c.q, room.c.scale) == (q.data_ptr(), scale.data_ptr())


def test_a_tensor_that_does_not_fit_is_refused_later_as_well(no_stream):
    room, x = rows(), torch.zeros(N, F)
    room._look(N, F)
    for name, value in (("q", torch.zeros(N, 32)), ("q", None), ("scale", None), ("scale", torch.zeros(N, **INT8)), ("columns", torch.zeros(2 * F)[::2])):
        assert refused(setattr, room, name, value)
        room._look(N, F)
    for name, value in (("q", torch.zeros(N, F, **INT8)), ("scale", torch.zeros(N - 1))):
        room = rows()
        room._look(N, F)
        setattr(room, name, value)
        assert refused(B.gnn_dequantize_rows, N, F, room, x), name


def test_a_copy_has_columns_of_its_own():
    room = rows()
    other = copy.copy(room)
    other.columns = torch.ones(F)
    assert not room.c.columns and other.c.columns == other.columns.data_ptr() and other.c.q == room.c.q


@pytest.mark.gpu
def test_xhat_with_gamma_given_later_is_the_norms_output():
    n, f = 300, 47
    rng = np.random.default_rng(3)
    X, gamma = (torch.from_numpy(rng.standard_normal(s).astype(np.float32)).cuda() for s in ((n, f), (f,)))
    Y, held, xhat8 = torch.empty_like(X), torch.empty_like(X), B.alloc_rows8(n, f)
    B.gnn_rms_norm_fwd(n, f, X, None, None, gamma, 1e-5, None, Y, xhat8, None)
    xhat8.columns = gamma
    B.gnn_dequantize_rows(n, f, xhat8, held)
    most = (X.abs().amax(1, keepdim=True) * torch.rsqrt((X * X).mean(1, keepdim=True) + 1e-5)) * gamma.abs() / 127
    assert bool(((held - Y).abs() <= 0.51 * most).all())
    other = torch.empty_like(X)
    xhat8.columns = None
    B.gnn_dequantize_rows(n, f, xhat8, other)
    assert torch.equal(other * gamma, held)
