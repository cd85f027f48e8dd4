"""The forms that the 4-bit linears and the packed cross-attention take, as host queries: what they refuse, and the rules' borders on a device
of 256 compute units."""
import ctypes as C

import pytest

from test_operators_abi_cpu import _caller


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


def test_refusals(m):
    lib, v = m.binding._lib, [C.byref(C.c_int32()) for _ in range(3)]
    linear = _caller(lib.ddit_linear_mx4_form, dict(epi=0, N=5, n=64, k=64, cus=0, rows=v[0], cols=v[1]))
    assert linear() == 0 and linear(N=0) == 0 and linear(epi=2) == 0
    for bad in (dict(epi=3), dict(epi=-1), dict(N=-1), dict(n=0), dict(k=0), dict(rows=None), dict(cols=None)):
        assert linear(**bad) == -1, bad
    for bad in (dict(n=60), dict(k=60), dict(N=1 << 26)):
        assert linear(**bad) == -2, bad
    cross = _caller(lib.ddit_cross_attn_packed_form, dict(B=2, q_rows=9, kv_rows=10, H=4, G=2, dh=64, cus=0, waves=v[0], parts=v[1], rows=v[2]))
    assert cross() == 0 and cross(q_rows=0, kv_rows=0) == 0
    for bad in (dict(B=0), dict(q_rows=-1), dict(kv_rows=-1), dict(H=0), dict(G=0), dict(G=3), dict(dh=0), dict(waves=None), dict(parts=None), dict(rows=None)):
        assert cross(**bad) == -1, bad
    for bad in (dict(dh=60), dict(dh=136), dict(B=1 << 20), dict(q_rows=1 << 31)):
        assert cross(**bad) == -2, bad


def test_linear_forms(m):
    form = lambda epi, N, n, k=1152: m.ddit_linear_mx4_form(epi, N, n, k, 256)
    for epi in (0, 1, 2):
        assert form(epi, 1, 6912) == form(epi, 16, 6912) == (16, 16)
        assert form(epi, 17, 2048) == form(epi, 32, 2048) == (32, 16) and form(epi, 17, 2056) == (64, 64) and form(epi, 33, 8) == (64, 64)
        assert form(epi, 128 * 255, 128) == (64, 64) and form(epi, 128 * 255 + 1, 128) == (128, 128)
    assert form(2, 256 * 511, 256) == (128, 128) and form(2, 256 * 511 + 1, 256) == (256, 256)
    assert form(0, 256 * 511 + 1, 256) == form(1, 256 * 511 + 1, 256) == (128, 128)
    assert form(2, 48600, 1152, 4608) == (256, 256) and form(1, 48600, 4608) == (128, 128)
    assert m.ddit_linear_mx4_form(2, 128 * 255, 128, 64, 64) == (256, 256)   # 64 compute units: 128 tiles of 256 are two rounds


def test_attention_forms(m):
    form = lambda *a: m.ddit_cross_attn_packed_form(*a, 256)
    assert form(3, 192, 900, 4, 4, 64)[:2] == (1, 1) and form(3, 193, 900, 4, 4, 64)[:2] == (8, 1)
    assert form(1, 8191, 300, 16, 16, 72)[0] == 8 and form(1, 8192, 300, 16, 16, 72)[0] == 12 and form(1, 8192, 300, 16, 16, 104)[0] == 8
    assert form(1, 1, 1023, 16, 16, 72) == (1, 1, 32) and form(1, 1, 1024, 16, 16, 72) == (1, 8, 32)
    assert form(4, 29, 7627, 16, 4, 128) == (1, 32, 32)
    assert form(1, 2000, 4096, 8, 8, 72) == (8, 4, 256)
    waves, parts, rows = form(2, 97200, 600, 16, 16, 72)
    assert (waves, parts) == (12, 1) and rows % 384 == 0
    # the workspace is enough for any number of key heads
    for totals in ((4, 29, 7627), (1, 2000, 4096), (2, 700, 1024)):
        need = m.ddit_cross_attn_packed_workspace_bytes(*totals, 16, 64)
        for G in (1, 2, 4, 8, 16):
            parts = form(*totals, 16, G, 64)[1]
            assert parts == 1 or parts * totals[1] * 16 * 66 * 4 <= need


def test_attention_forms_of_a_smaller_device(m):
    """Two rounds of the chip are two of the device's: from 512 rows a compute unit on, counted over the key heads."""
    for cus in (32, 64, 256):
        form = lambda rows, dh: m.ddit_cross_attn_packed_form(1, rows, 300, 16, 16, dh, cus)[0]
        assert form(32 * cus - 1, 72) == 8 and form(32 * cus, 72) == 12 and form(32 * cus, 104) == 8
