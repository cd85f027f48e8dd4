"""Sizes whose launch would hold 2^32 work-items or more, which a launch cannot: refused by name before anything reaches the device, so no
GPU is needed."""
import pytest

from test_operators_abi_cpu import P, _caller


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


def test_packed_attention_with_more_workgroups_than_a_launch_holds(m):
    """2^23 queries of 128 heads for 65536 requests: 87381 + 65536 slots a head, 768 threads each."""
    call = _caller(m.binding._lib.ddit_cross_attn_packed_fwd, dict(
        q=P(0x1000), ld_q=1024, q_off=P(0x2000), k=None, v=None, ld_kv=1024, kv_off=P(0x5000), mask=None, B=65536, q_rows=1 << 23, kv_rows=0, H=128, G=128, dh=8,
        scale=0.125, o=P(0x6000), ld_o=1024, lse=None, ws=None, bytes=0, stream=None))
    assert call() == -2 and "workgroups" in m.ddit_last_error()
    assert call(dh=128, ld_q=16384, ld_kv=16384, ld_o=16384) == -2
