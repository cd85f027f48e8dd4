"""The logarithms that the packed attention of a sublayer leaves beside its outputs, against float64 from the queries and keys in memory."""
import pytest
import torch

from test_gpu_cross_packed import reference
from test_gpu_operators_together import Sublayer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,states,D,H,dh", [([300, 77, 1], [30, 0, 120], 1152, 16, 72), ([9, 3], [700, 900], 256, 4, 64), ([2000, 1500], [300, 41], 1152, 16, 72)])
def test_lse_of_a_sublayer(tokens, states, D, H, dh):
    import paper_2506_13497_amd as m
    s = Sublayer(m, tokens, states, D, H, dh, 3)
    for _ in range(2):
        s.lse.fill_(float("nan"))
        s.run()
        torch.cuda.synchronize()
        _, _, lse, el = reference(s.q, s.kv[:, :s.A], s.kv[:, s.A:], s.q_off.tolist(), s.kv_off.tolist(), None, H, H, dh, dh ** -0.5)
        none = lse == -float("inf")
        assert torch.equal(s.lse == -float("inf"), none)
        assert ((s.lse.double() - lse).abs()[~none] <= el[~none]).all()
        s.fill()
