"""Norms around a branch where four wavefronts share a row and a workgroup takes several rows, which end samples in between: the rows' sums meet
in the same two places in turn, and the vectors of a sample are replaced by the next one's.  Tolerances as in the module that holds the reference."""
import pytest
import torch

from test_gpu_branch_norms import _check, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


# the grid is at most eight workgroups a CU, 2048 of them: two to five rows each
@pytest.mark.parametrize("N,D,tps", [(9001, 2056, 3001), (9001, 2056, 3), (6000, 4096, 1), (4999, 4104, 2), (5000, 8192, 1700), (2049, 8192, 5)])
@pytest.mark.parametrize("kind", [0, 1])
def test_several_rows_a_workgroup(m, N, D, tps, kind):
    t = _inputs(N, D, tps, N + D)
    want = _check(m, t, kind, 2, 1, True, 0.875, tps)
    _check(m, t, kind, 2, 1, True, 0.875, tps, in_place=True)
    # the stream alone: one sum a row (RMS), or two
    x_out = torch.full_like(t["x"], float("nan"))
    m.ddit_branch_norms_fwd(kind, t["f"], D, t["g_post"], t["x"], 0.875, t["table"], t["c6"], 2, x_out, t["g_pre"], t["next_table"], -1, tps, 1e-6, None, 0)
    torch.cuda.synchronize()
    assert torch.equal(x_out, want[0])


@pytest.mark.parametrize("kind", [0, 1])
def test_the_same_bits_every_time(m, kind):
    t = _inputs(9001, 2056, 70, 5)
    a = _check(m, t, kind, 5, 0, True, 1.0, 70)
    for _ in range(3):
        b = _check(m, t, kind, 5, 0, True, 1.0, 70)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1].view(torch.int16), b[1].view(torch.int16))
