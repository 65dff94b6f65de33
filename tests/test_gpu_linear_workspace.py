"""The products within the workspace that they ask for, on both sides of the rows from which on X in 8 bits is read as it is, and where
rows are padded: nothing behind it is written, and the results are right."""
import pytest
import torch

from paper_2308_12093_amd import binding as B
from tests import test_gpu_linear as linear

pytestmark = pytest.mark.gpu

BEHIND = 4 << 20


@pytest.fixture
def guarded(monkeypatch):
    made = []

    def workspace(c, back):
        nbytes = B.gnn_linear_workspace_bytes(back, c.n, c.m, c.k)
        room = torch.full((nbytes + BEHIND,), 255, dtype=torch.uint8, device="cuda")
        made.append(room[nbytes:])
        return room[:nbytes]

    monkeypatch.setattr(linear, "workspace", workspace)
    return made


@pytest.mark.parametrize("by", [0, 1])
@pytest.mark.parametrize("n,m,k", [(1119, 512, 1024), (1121, 512, 1024), (1920, 512, 1024), (1921, 512, 1024), (1922, 512, 1024),
                                   (32640, 128, 256), (32641, 128, 256), (32767, 65, 70), (32769, 65, 70), (10880, 300, 131), (10881, 300, 131),
                                   (10880, 203, 259), (10881, 203, 259), (11009, 203, 259), (40000, 203, 47), (40000, 47, 300), (40000, 35, 33)])
def test_nothing_behind_the_workspace_is_written(guarded, n, m, k, by):
    linear.every_way(linear.Case(n, m, k, "silu"), by)
    assert len(guarded) >= 6 and all(bool((end == 255).all()) for end in guarded)
