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


def test_one_row_of_all_panels(m):
    """2^24 panels of one row: a workgroup of 256 threads each."""
    lib = m.binding._lib
    for fn, args in ((lib.ddit_mx4_quantize, dict(x=P(0x1000), ld=1 << 31, rows=1, k=(1 << 31) - 8, codes=P(0x2000), scales=P(0x3000), stream=None)),
                     (lib.ddit_mx4_dequantize, dict(codes=P(0x2000), scales=P(0x3000), rows=1, k=(1 << 31) - 8, x=P(0x1000), ld=1 << 31, stream=None))):
        call = _caller(fn, args)
        assert call() == -2 and "panels" in m.ddit_last_error()
        assert call(rows=0) == 0
