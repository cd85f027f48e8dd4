"""The 4-bit linears' tiles where a workgroup makes several of them, with one to a few panels of k: the stream of loads then runs on into the next
tiles, several ahead.  The tile that a case is meant for is asked for.  Tolerances as in the module that holds the reference."""
import pytest
import torch

from test_gpu_mx4 import _check_linear, _problem, _same_values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


@pytest.mark.parametrize("k", [8, 128, 136, 392])
def test_residual_in_tiles_of_256(m, k):
    """570 tiles for 256 workgroups: one to four panels, samples that end inside a wavefront's 128 rows, ragged in both directions."""
    N, n = 29001, 1160
    assert m.ddit_linear_mx4_form(2, N, n, k) == (256, 256)
    _check_linear(m, N, n, k, 2, seed=k, tps=7001)
    _check_linear(m, N, n, k, 2, seed=k + 1, tps=70, gate_row=0, bias=False, ld_out=1176)
    _check_linear(m, N, n, k, 2, seed=k + 2, gate_row=-1, copy=False)
    a = _check_linear(m, N, n, k, 2, seed=k + 3, tps=9000)
    b = _check_linear(m, N, n, k, 2, seed=k + 3, tps=9000, codes=True)
    assert _same_values(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("N,n,k,tps", [(29001, 1160, 264, 1000), (33000, 1152, 4608, 16500)])
def test_residual_in_tiles_of_256_in_place(m, N, n, k, tps):
    assert m.ddit_linear_mx4_form(2, N, n, k) == (256, 256)
    a = _check_linear(m, N, n, k, 2, seed=6, tps=tps)
    t = _problem(m, N, n, k, 6)
    c6 = t["c6"](tps)
    x, out = t["x"].clone(), torch.empty((N, n), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(m.ddit_linear_mx4_workspace_bytes(N, n, k), dtype=torch.uint8, device="cuda")
    m.ddit_linear_mx4_fwd(2, t["u"], k, t["wc"], t["ws"], t["bias"], N, n, k, out, n, ws, resid=x, resid_out=x, ada_table=t["table"], c6=c6, gate_row=5,
                          tokens_per_sample=tps)
    torch.cuda.synchronize()
    assert torch.equal(x, a[1][:N]) and _same_values(out, a[0][:N])


@pytest.mark.parametrize("epi,N,n", [(0, 20003, 1160), (1, 20003, 1160), (2, 9001, 1160)])
@pytest.mark.parametrize("k", [8, 128, 136, 264, 392])
def test_several_tiles_of_128(m, epi, N, n, k):
    """More tiles than workgroups that fit the chip (three a CU, the residual update two)."""
    assert m.ddit_linear_mx4_form(epi, N, n, k) == (128, 128)
    _check_linear(m, N, n, k, epi, seed=k, tps=N // 3)


@pytest.mark.parametrize("epi", [0, 1, 2])
@pytest.mark.parametrize("k", [8, 128, 136, 264, 392])
def test_several_tiles_of_64(m, epi, k):
    """900 tiles for 768 workgroups; panels go in pairs, the last one alone where their number is odd."""
    N, n = 3195, 1144
    assert m.ddit_linear_mx4_form(epi, N, n, k) == (64, 64)
    _check_linear(m, N, n, k, epi, seed=k, tps=100)
