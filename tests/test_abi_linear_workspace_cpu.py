"""What the products ask for as scratch: no launch, so no GPU is needed."""
import pytest

from paper_2308_12093_amd import binding as B


@pytest.mark.parametrize("n,m,k", [(1 << 16, 512, 1024), (1 << 16, 512, 2048), (1 << 18, 1024, 256), (1 << 17, 128, 256)])
def test_backward_has_room_for_no_array_that_it_does_not_form(n, m, k):
    """D in floats, and 128 MB: partial sums of dW (512 blocks of 128 x 256 floats, 67 MB, or one array where that is more), the weights'
    parts, largest magnitudes and the rows in 8 bits that are brought to floats, where they are few.  No n x m floats (67 MB and more), and
    not a second time n x k."""
    assert B.gnn_linear_workspace_bytes(True, n, m, k) <= 4 * n * k + (128 << 20)


def test_forward_has_room_for_rows_only_where_it_pads_them():
    n, m = 1 << 16, 203
    assert B.gnn_linear_workspace_bytes(False, n, m, 47) < 4 << 20
    assert B.gnn_linear_workspace_bytes(False, n, m, 259) > 4 * n * m


@pytest.mark.parametrize("m,k", [(512, 1024), (1024, 256), (128, 256), (128, 129), (65, 70), (300, 131), (203, 259), (47, 300), (203, 47), (64, 65), (35, 33),
                                 (31, 200), (4, 4), (130, 2048)])
def test_a_workspace_serves_fewer_rows(m, k):
    """On both sides of every number of rows where another kernel takes over."""
    least = [(-(-256 // tiles) - 1) * 128 for tiles in range(1, 257)]
    near = {n + d for n in least + [32 * t for t in range(1, 2000, 7)] for d in (-1, 0, 1, 2, 33)}
    rows = sorted(n for n in near | set(range(30600, 34000)) | {1 << p for p in range(24)} if n > 0)
    for back in (0, 1):
        sizes = [B.gnn_linear_workspace_bytes(back, n, m, k) for n in rows]
        fall = [(n, a, b) for n, a, b in zip(rows[1:], sizes, sizes[1:]) if b < a]
        assert not fall, fall[:3]
