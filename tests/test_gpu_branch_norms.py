"""Norms on both sides of a residual branch against float64, at the borders of the kernel's forms (few rows, 512, 1280, 2048, 4096 and
8192 features), with every option on and off.

Tolerances.  One unit u = 2^-24 is half a step of fp32 relative to the value.  A row's sums pass at most 8 x 4 additions in a lane and
8 across lanes and wavefronts: a mean is off by at most 40 u mean|v|, a sum of squares by 40 u of itself, so n = Norm(v) is off by at most
64 u (a + |n|) with a = mean|v| / sqrt(var + eps), which adds 20 u for the subtraction, the root and the products.  The stream adds 4 u of
each of its two terms; bf16 rounds by at most 2^-8 of the value."""
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


def _norm64(v, kind, eps):
    """-> Norm(v), and the largest error that fp32 may make in it"""
    c = v - v.mean(1, keepdim=True) if kind == 0 else v
    rstd = ((c * c).mean(1, keepdim=True) + eps).rsqrt()
    n = c * rstd
    return n, 64 * U * (v.abs().mean(1, keepdim=True) * rstd + n.abs()), rstd


def _reference(kind, f, g_post, x, r, table, c6, gate_row, g_pre, next_table, which, tps, eps):
    N, D = x.shape
    at = torch.arange(N, device=x.device) // tps
    c = None if c6 is None else c6.double().view(-1, 6, D)
    one = torch.ones((), dtype=torch.float64, device=x.device)
    gp = one if g_post is None else g_post.double()
    gate = one if gate_row < 0 else (table.double()[gate_row] + c[:, gate_row])[at]
    s = one if g_pre is None else g_pre.double()
    t = one * 0
    if which >= 0:
        s = s * (1 + (next_table.double()[3 * which + 1] + c[:, 3 * which + 1])[at])
        t = (next_table.double()[3 * which] + c[:, 3 * which])[at]
    n, en, _ = _norm64(f.double(), kind, eps)
    w = gate * gp
    y = r * x.double() + w * n
    ey = w.abs() * en + 4 * U * ((r * x.double()).abs() + (w * n).abs())
    n2, en2, rstd = _norm64(y, kind, eps)
    h = n2 * s + t
    # an error of y moves its own feature, and through mean and variance every feature of the row
    moved = rstd * (ey + (1 + n2.abs()) * ey.amax(1, keepdim=True))
    eh = 2.0 ** -8 * h.abs() + s.abs() * (en2 + moved) + 4 * U * ((n2 * s).abs() + t.abs())
    return y, ey, h, eh


def _inputs(N, D, tps, seed, scale=1.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(*s, device="cuda", generator=g)
    B = (N + tps - 1) // tps
    return dict(f=(draw(N, D) * scale + 0.3).bfloat16(), x=draw(N, D) * 3 + 0.5, g_post=(1 + 0.2 * draw(D)).bfloat16(),
                g_pre=(1 + 0.2 * draw(D)).bfloat16(), table=draw(6, D) * 0.5, next_table=draw(6, D) * 0.5, c6=draw(B, 6 * D) * 0.5)


def _check(m, t, kind, gate_row, which, affine, r, tps, eps=1e-6, in_place=False):
    N, D = t["x"].shape
    gp, gq = (t["g_post"], t["g_pre"]) if affine else (None, None)
    y, ey, h, eh = _reference(kind, t["f"], gp, t["x"], r, t["table"], t["c6"], gate_row, gq, t["next_table"], which, tps, eps)
    x = t["x"].clone()
    x_out = x if in_place else torch.full_like(x, float("nan"))
    out = torch.full((N, D), float("nan"), dtype=torch.bfloat16, device="cuda")
    m.ddit_branch_norms_fwd(kind, t["f"], D, gp, x, r, t["table"], t["c6"], gate_row, x_out, gq, t["next_table"], which, tps, eps, out, D)
    torch.cuda.synchronize()
    assert ((x_out.double() - y).abs() <= ey).all()
    assert ((out.double() - h).abs() <= eh).all()
    if not in_place:
        assert torch.equal(x, t["x"])
    return x_out, out


@pytest.mark.parametrize("N,D,tps", [(1, 8, 1), (1, 1152, 1), (3, 64, 2), (5, 512, 5), (7, 520, 2), (1023, 1152, 1023), (1025, 1152, 400),
                                     (2100, 504, 1), (4099, 512, 4099), (2047, 1280, 700), (1500, 1288, 1500), (1030, 2048, 1030), (37, 2056, 9),
                                     (300, 4096, 150), (33, 4104, 33), (130, 8192, 65), (9001, 1152, 3001), (2, 8192, 1)])
@pytest.mark.parametrize("kind", [0, 1])
def test_borders_of_the_forms(m, N, D, tps, kind):
    _check(m, _inputs(N, D, tps, N * 7 + D), kind, 2, 1, True, 0.875, tps)


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("gate_row", [-1, 0, 5])
@pytest.mark.parametrize("which", [-1, 0, 1])
@pytest.mark.parametrize("affine", [False, True])
def test_every_option(m, kind, gate_row, which, affine):
    for N, D, tps in [(29, 1152, 10), (1300, 136, 500)]:
        _check(m, _inputs(N, D, tps, 5 + N), kind, gate_row, which, affine, 1.0, tps, in_place=gate_row == 5)


def test_one_form_gives_the_bits_of_the_other_samples(m):
    """A row's result does not depend on how many rows the call has, where the form is the same."""
    t = _inputs(9000, 1152, 9000, 3)
    a = _check(m, t, 0, 2, 0, True, 1.0, 9000)
    small = {k: (v[:5000].contiguous() if k in ("f", "x") else v) for k, v in t.items()}
    b = _check(m, small, 0, 2, 0, True, 1.0, 5000)
    assert torch.equal(a[0][:5000], b[0]) and torch.equal(a[1][:5000].view(torch.int16), b[1].view(torch.int16))


@pytest.mark.parametrize("N", [50, 3000])
def test_strides_rows_behind_and_the_stream_alone(m, N):
    D, ld_f, ld_o = 1152, 1160, 2304
    t = _inputs(N, D, N, 11)
    want = _check(m, t, 1, 2, 1, True, 1.0, N)
    wide = torch.full((N + 3, ld_f), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:N, :D] = t["f"]
    out = torch.full((N + 3, ld_o), -7.0, dtype=torch.bfloat16, device="cuda")
    xo = torch.full((N + 3, D), -7.0, device="cuda")
    call = lambda h: m.ddit_branch_norms_fwd(1, wide, ld_f, t["g_post"], t["x"], 1.0, t["table"], t["c6"], 2, xo, t["g_pre"], t["next_table"],
                                             1 if h is not None else -1, N, 1e-6, h, ld_o)
    call(out)
    torch.cuda.synchronize()
    assert torch.equal(xo[:N], want[0]) and torch.equal(out[:N, :D].contiguous().view(torch.int16), want[1].view(torch.int16))
    assert (xo[N:] == -7).all() and (out[N:] == -7).all() and (out[:, D:] == -7).all()
    xo.fill_(-7.0)
    call(None)
    torch.cuda.synchronize()
    assert torch.equal(xo[:N], want[0]) and (xo[N:] == -7).all()


@pytest.mark.parametrize("N,D", [(40, 1152), (2000, 256), (64, 4096)])
def test_a_bad_row_stays_alone(m, N, D):
    t = _inputs(N, D, N, 17)
    want = _check(m, t, 0, 2, 1, True, 1.0, N)
    for at, what in ((5, float("nan")), (9, float("inf"))):
        t["f"][at, 3] = what
    x_out, out = torch.empty_like(t["x"]), torch.empty_like(t["f"])
    m.ddit_branch_norms_fwd(0, t["f"], D, t["g_post"], t["x"], 1.0, t["table"], t["c6"], 2, x_out, t["g_pre"], t["next_table"], 1, N, 1e-6, out, D)
    torch.cuda.synchronize()
    good = torch.ones(N, dtype=torch.bool, device="cuda")
    good[[5, 9]] = False
    assert torch.equal(x_out[good], want[0][good]) and torch.equal(out[good].view(torch.int16), want[1][good].view(torch.int16))
    assert x_out[~good].isnan().all() and out[~good].isnan().all()


def test_constant_and_zero_rows_and_a_large_eps(m):
    t = _inputs(64, 1152, 64, 19)
    t["f"][3] = 0
    t["f"][4] = 2.0      # no variance: a LayerNorm gives zeros, and the stream alone remains
    _check(m, t, 0, 2, 1, True, 1.0, 64)
    _check(m, t, 1, 2, 1, True, 1.0, 64)
    _check(m, t, 1, 2, 1, True, -2.0, 64, eps=0.5)
    _check(m, t, 0, -1, -1, False, 0.0, 64)


def test_captured_and_on_another_stream(m):
    N, D = 700, 1152
    t = _inputs(N, D, 350, 23)
    x_out, out = torch.empty_like(t["x"]), torch.empty_like(t["f"])
    call = lambda: m.ddit_branch_norms_fwd(0, t["f"], D, t["g_post"], t["x"], 1.0, t["table"], t["c6"], 2, x_out, t["g_pre"], t["next_table"], 0,
                                           350, 1e-6, out, D)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in (1, 2, 3):
        new = _inputs(N, D, 350, seed)
        for k in t:
            t[k].copy_(new[k])
        graph.replay()
        torch.cuda.synchronize()
        want = _check(m, t, 0, 2, 0, True, 1.0, 350)
        assert torch.equal(x_out, want[0]) and torch.equal(out.view(torch.int16), want[1].view(torch.int16))
