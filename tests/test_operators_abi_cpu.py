"""What the norms around a branch, the 4-bit linears and the packed cross-attention refuse, and their host-only queries: every check
comes before anything is enqueued, so no GPU is needed."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


def P(v):
    return C.c_void_p(v)


def _caller(fn, args):
    """fn with these arguments, some replaced by name."""
    def call(**kw):
        assert set(kw) <= set(args)
        return fn(*[kw.get(n, v) for n, v in args.items()])
    return call


def test_branch_norms_refusals(m):
    call = _caller(m.binding._lib.ddit_branch_norms_fwd, dict(
        norm=0, f=P(0x1000), ld_f=64, g_post=None, x=P(0x2000), r=1.0, gate_table=P(0x3000), c6=P(0x4000), gate_row=2, x_out=P(0x5000), g_pre=None,
        next_table=P(0x6000), which=1, N=0, tps=1, D=64, eps=1e-6, out=P(0x7000), ld_out=64, stream=None))
    assert call() == 0 and call(x_out=P(0x2000)) == 0          # zero tokens: checked, and nothing done
    assert call(gate_row=-1, which=-1, gate_table=None, next_table=None, c6=None) == 0
    assert call(which=-1, out=None, ld_out=0) == 0
    assert call(f=None, x=None, x_out=None, out=None) == 0     # nothing has no address
    for bad in (dict(norm=2), dict(norm=-1), dict(N=3, f=None), dict(N=3, x=None), dict(N=3, x_out=None), dict(N=-1), dict(tps=0), dict(D=0), dict(eps=0.0),
                dict(eps=float("nan")), dict(gate_row=6), dict(which=2), dict(r=float("inf")), dict(r=float("nan")), dict(ld_f=56), dict(ld_out=56),
                dict(gate_table=None), dict(c6=None), dict(next_table=None), dict(c6=None, which=-1), dict(N=3, out=None)):
        assert call(**bad) == -1, bad
        assert m.ddit_last_error()
    for bad in (dict(D=60, ld_f=64), dict(D=8200, ld_f=8200, ld_out=8200), dict(N=1 << 50)):
        assert call(**bad) == -2, bad
    for bad in (dict(ld_f=68), dict(ld_out=68), dict(f=P(0x1008)), dict(x=P(0x2004)), dict(x_out=P(0x5008)), dict(g_post=P(0x8)), dict(g_pre=P(0x8)),
                dict(gate_table=P(0x3004)), dict(c6=P(0x4008)), dict(next_table=P(0x6008)), dict(out=P(0x7008))):
        assert call(**bad) == -4, bad


def test_mx4_sizes_and_refusals(m):
    lib = m.binding._lib
    assert m.ddit_mx4_bytes(0, 8) == (0, 0) and m.ddit_mx4_bytes(3, 8) == (192, 12) and m.ddit_mx4_bytes(5, 1152) == (5 * 9 * 64, 5 * 9 * 4)
    assert m.ddit_mx4_bytes(5, 1160) == (5 * 10 * 64, 5 * 10 * 4)
    assert m.ddit_linear_mx4_workspace_bytes(0, 64, 64) == 0
    for N, n, k in [(1, 8, 8), (300, 2304, 1152), (48600, 1152, 4608)]:
        c, s = m.ddit_mx4_bytes(N, k)
        assert c + s <= m.ddit_linear_mx4_workspace_bytes(N, n, k) <= c + s + 512
    size = C.c_size_t()
    for rows, k, code in [(-1, 64, -1), (1, 0, -1), (1, 12, -2), (1 << 25, 128, -2), ((1 << 31), 8, -2), (1 << 62, 1 << 30, -2)]:
        assert lib.ddit_mx4_bytes(rows, k, C.byref(size), C.byref(size)) == code, (rows, k)
        assert lib.ddit_linear_mx4_workspace_bytes(rows, 64, k, C.byref(size)) == code
    assert lib.ddit_mx4_bytes(1, 8, None, C.byref(size)) == -1 and lib.ddit_mx4_bytes(1, 8, C.byref(size), None) == -1
    assert lib.ddit_linear_mx4_workspace_bytes(1, 0, 8, C.byref(size)) == -1 and lib.ddit_linear_mx4_workspace_bytes(1, 8, 8, None) == -1
    q = _caller(lib.ddit_mx4_quantize, dict(x=P(0x1000), ld=64, rows=0, k=64, codes=P(0x2000), scales=P(0x3000), stream=None))
    d = _caller(lib.ddit_mx4_dequantize, dict(codes=P(0x2000), scales=P(0x3000), rows=0, k=64, x=P(0x1000), ld=64, stream=None))
    for call in (q, d):
        assert call() == 0 and call(x=None, codes=None, scales=None) == 0
        for bad in (dict(rows=3, x=None), dict(rows=3, codes=None), dict(rows=3, scales=None), dict(rows=-1), dict(k=0), dict(ld=56)):
            assert call(**bad) == -1, bad
        for bad in (dict(k=12), dict(rows=1 << 26)):
            assert call(**bad) == -2, bad
        for bad in (dict(ld=68), dict(x=P(0x1008)), dict(codes=P(0x2008)), dict(scales=P(0x3004))):
            assert call(**bad) == -4, bad


def test_linear_mx4_refusals(m):
    lib = m.binding._lib
    tail = dict(wc=P(0x3000), ws=P(0x4000), bias=None, N=0, n=64, k=64, out=P(0x5000), ld_out=64, resid=None, resid_out=None, table=None, c6=None,
                gate_row=-1, tps=1)
    dense = _caller(lib.ddit_linear_mx4_fwd, dict(epi=0, u=P(0x1000), ld_u=64, **tail, workspace=None, bytes=0, stream=None))
    coded = _caller(lib.ddit_linear_mx4_codes_fwd, dict(epi=0, u=P(0x1000), us=P(0x2000), **tail, stream=None))
    resid = dict(epi=2, resid=P(0x6000), resid_out=P(0x7000))
    for call in (dense, coded):
        assert call() == 0 and call(**resid) == 0 and call(**resid, out=None, ld_out=0) == 0
        assert call(**resid, gate_row=5, table=P(0x8000), c6=P(0x9000)) == 0
        assert call(u=None, out=None) == 0 and call(epi=2, u=None, out=None) == 0
        for bad in (dict(epi=3), dict(epi=-1), dict(N=3, u=None), dict(wc=None), dict(ws=None), dict(N=-1), dict(n=0), dict(k=0), dict(N=3, out=None), dict(ld_out=56),
                    dict(resid, N=3, resid=None), dict(resid, N=3, resid_out=None), dict(resid, gate_row=2), dict(resid, gate_row=6, table=P(0x8000), c6=P(0x9000)),
                    dict(resid, gate_row=2, table=P(0x8000)), dict(resid, gate_row=2, table=P(0x8000), c6=P(0x9000), tps=0)):
            assert call(**bad) == -1, bad
        for bad in (dict(n=60), dict(k=60), dict(N=1 << 26), dict(n=1 << 26, ld_out=1 << 26), dict(n=1 << 24, ld_out=1 << 24), dict(ld_out=1 << 25)):
            assert call(**bad) == -2, bad
        for bad in (dict(ld_out=68), dict(u=P(0x1008)), dict(wc=P(0x3008)), dict(ws=P(0x4004)), dict(bias=P(0x8)), dict(out=P(0x5008)),
                    dict(resid, resid=P(0x6008)), dict(resid, resid_out=P(0x7008)), dict(resid, gate_row=0, table=P(0x8004), c6=P(0x9000)),
                    dict(resid, gate_row=0, table=P(0x8000), c6=P(0x9004))):
            assert call(**bad) == -4, bad
    assert coded(N=3, us=None) == -1 and coded(us=P(0x2008)) == -4
    assert dense(ld_u=56) == -1 and dense(ld_u=68) == -4
    need = m.ddit_linear_mx4_workspace_bytes(5, 64, 64)
    assert dense(N=5) == -3 and dense(N=5, workspace=P(0x10000), bytes=need - 1) == -3 and str(need) in m.ddit_last_error()
    assert dense(N=5, workspace=P(0x10010), bytes=need) == -4


def test_cross_packed_refusals(m):
    lib = m.binding._lib
    call = _caller(lib.ddit_cross_attn_packed_fwd, dict(
        q=P(0x1000), ld_q=256, q_off=P(0x2000), k=P(0x3000), v=P(0x4000), ld_kv=128, kv_off=P(0x5000), mask=None, B=2, q_rows=0, kv_rows=10, H=4, G=2, dh=64,
        scale=0.125, o=P(0x6000), ld_o=256, lse=None, ws=None, bytes=0, stream=None))
    assert call() == 0 and call(mask=P(0x7001), lse=P(0x8004)) == 0
    assert call(q=None, o=None) == 0 and call(kv_rows=0, k=None, v=None) == 0
    for bad in (dict(q_rows=3, q=None), dict(k=None), dict(v=None), dict(q_rows=3, o=None), dict(q_off=None), dict(kv_off=None), dict(B=0), dict(q_rows=-1), dict(kv_rows=-1), dict(H=0),
                dict(G=0), dict(G=3), dict(dh=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=2e38), dict(ld_q=248),
                dict(ld_kv=120), dict(ld_o=248)):
        assert call(**bad) == -1, bad
    for bad in (dict(dh=60), dict(dh=136, ld_q=1024, ld_kv=1024, ld_o=1024), dict(B=1 << 20), dict(q_rows=1 << 31), dict(kv_rows=1 << 31), dict(H=1 << 17), dict(ld_o=1 << 22), dict(ld_q=1 << 22), dict(ld_kv=1 << 22)):
        assert call(**bad) == -2, bad
    for bad in (dict(ld_q=260), dict(ld_kv=132), dict(ld_o=260), dict(q=P(0x1008)), dict(k=P(0x3008)), dict(v=P(0x4002)), dict(o=P(0x6008)), dict(q_off=P(0x2002)),
                dict(kv_off=P(0x5001)), dict(lse=P(0x8002))):
        assert call(**bad) == -4, bad
    # a few queries against long encodings: parts of the keys, whose sums need room
    few = dict(q_rows=10, kv_rows=8000)
    need = m.ddit_cross_attn_packed_workspace_bytes(2, 10, 8000, 4, 64)
    assert need > 0 and m.ddit_cross_attn_packed_workspace_bytes(2, 100000, 8000, 4, 64) == 0 and m.ddit_cross_attn_packed_workspace_bytes(2, 0, 8000, 4, 64) == 0
    assert call(**few) == -3 and call(**few, ws=P(0x10000), bytes=need - 1) == -3 and str(need) in m.ddit_last_error()
    assert call(**few, ws=P(0x10010), bytes=need) == -4
    size = C.c_size_t()
    assert lib.ddit_cross_attn_packed_workspace_bytes(0, 1, 1, 1, 64, C.byref(size)) == -1
    assert lib.ddit_cross_attn_packed_workspace_bytes(1, 1, 1, 1, 60, C.byref(size)) == -2
    assert lib.ddit_cross_attn_packed_workspace_bytes(1, 1, 1, 1, 64, None) == -1
