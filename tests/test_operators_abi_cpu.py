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
    for bad in (dict(norm=2), dict(norm=-1), dict(f=None), dict(x=None), dict(x_out=None), dict(N=-1), dict(tps=0), dict(D=0), dict(eps=0.0),
                dict(eps=float("nan")), dict(gate_row=6), dict(which=2), dict(r=float("inf")), dict(r=float("nan")), dict(ld_f=56), dict(ld_out=56),
                dict(gate_table=None), dict(c6=None), dict(next_table=None), dict(c6=None, which=-1), dict(out=None)):
        assert call(**bad) == -1, bad
        assert m.ddit_last_error()
    for bad in (dict(D=60, ld_f=64), dict(D=8200, ld_f=8200, ld_out=8200), dict(N=1 << 50)):
        assert call(**bad) == -2, bad
    for bad in (dict(ld_f=68), dict(ld_out=68), dict(f=P(0x1008)), dict(x=P(0x2004)), dict(x_out=P(0x5008)), dict(g_post=P(0x8)), dict(g_pre=P(0x8)),
                dict(gate_table=P(0x3004)), dict(c6=P(0x4008)), dict(next_table=P(0x6008)), dict(out=P(0x7008))):
        assert call(**bad) == -4, bad
