"""Arrays whose bytes lie further than 2^31 from their start, in every operand that has rows: strided activations and outputs, the fp32 stream,
queries, states.  Only a few rows are looked at, the first and the last and those around 2^31 and 2^32 bytes; the memory between strided rows is
never touched.  Tolerances as in the modules that hold the references."""
import math

import pytest
import torch

from test_gpu_branch_norms import _inputs, _reference
from test_gpu_cross_packed import offsets, reference as cross_reference
from test_gpu_mx4 import U, decode64, encode64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


@pytest.fixture(autouse=True)
def _give_back():
    yield
    torch.cuda.empty_cache()


def spread(rows, cols, ld, values=None):
    """bf16 [rows, cols] in rows of ld elements; the last byte is past 2^31."""
    assert rows * ld * 2 > 1 << 31
    at = torch.empty(((rows - 1) * ld + cols,), dtype=torch.bfloat16, device="cuda").as_strided((rows, cols), (ld, 1))
    if values is None:
        at.fill_(-7.0)
    else:
        at.copy_(values)
    return at


def some_rows(N, bytes_a_row):
    at = {0, 1, N - 1}
    for border in (1 << 31, 1 << 32):
        at |= {border // bytes_a_row + d for d in (-1, 0, 1)}
    return torch.tensor(sorted(r for r in at if 0 <= r < N), device="cuda")


def test_norms_of_strided_rows(m):
    N, D, ld = 700, 1152, 1 << 21
    t = _inputs(N, D, 300, 1)
    f, out = spread(N, D, ld, t["f"]), spread(N, D, ld)
    x_out = torch.empty_like(t["x"])
    m.ddit_branch_norms_fwd(0, f, ld, t["g_post"], t["x"], 1.0, t["table"], t["c6"], 2, x_out, t["g_pre"], t["next_table"], 1, 300, 1e-6, out, ld)
    torch.cuda.synchronize()
    y, ey, h, eh = _reference(0, t["f"], t["g_post"], t["x"], 1.0, t["table"], t["c6"], 2, t["g_pre"], t["next_table"], 1, 300, 1e-6)
    assert ((x_out.double() - y).abs() <= ey).all() and ((out.double() - h).abs() <= eh).all()


@pytest.mark.parametrize("N,D", [(140001, 8192), (600001, 1152)])
def test_norms_of_a_long_stream(m, N, D):
    """The stream, read and written, and for the wider one f and out too: past 2^32 bytes."""
    g = torch.Generator(device="cuda").manual_seed(2)
    t = _inputs(1, D, 1, 2)
    f = torch.empty((N, D), dtype=torch.bfloat16, device="cuda").normal_(0.3, 1.5, generator=g)
    x = torch.empty((N, D), device="cuda").normal_(0.5, 3.0, generator=g)
    at = some_rows(N, 4 * D)
    rows = {"f": f[at].clone(), "x": x[at].clone()}
    out = torch.empty_like(f)
    m.ddit_branch_norms_fwd(1, f, D, t["g_post"], x, 1.0, t["table"], t["c6"], 2, x, t["g_pre"], t["next_table"], 1, N, 1e-6, out, D)
    torch.cuda.synchronize()
    y, ey, h, eh = _reference(1, rows["f"], t["g_post"], rows["x"], 1.0, t["table"], t["c6"], 2, t["g_pre"], t["next_table"], 1, len(at), 1e-6)
    assert ((x[at].double() - y).abs() <= ey).all() and ((out[at].double() - h).abs() <= eh).all()


def _weights(m, n, k, g):
    P = (k + 127) // 128
    W = (0.05 * torch.randn(n, k, device="cuda", generator=g)).bfloat16()
    c, s = torch.empty((P, n, 64), dtype=torch.uint8, device="cuda"), torch.empty((P, n, 4), dtype=torch.uint8, device="cuda")
    m.ddit_mx4_quantize(W, k, n, k, c, s)
    torch.cuda.synchronize()
    return c, s, decode64(c, s, k)


def _product(u, W64, k):
    u64 = decode64(*(t.cuda() for t in encode64(u.cpu())), k)
    return u64 @ W64.t().contiguous(), (4 * ((k + 127) // 128) + 20) * U * (u64.abs() @ W64.abs().t().contiguous())


@pytest.mark.parametrize("N", [90, 20])
def test_conversions_and_linears_of_strided_rows(m, N):
    """Rows 2^24 elements apart: 90 of them in tiles, 20 in the launch of few tokens with 2^26 between them."""
    k, n, ld = 328, 264, (1 << 24) if N == 90 else (1 << 26)
    g = torch.Generator(device="cuda").manual_seed(3)
    u = spread(N, k, ld, torch.randn(N, k, device="cuda", generator=g))
    codes, scales = torch.empty((3, N, 64), dtype=torch.uint8, device="cuda"), torch.empty((3, N, 4), dtype=torch.uint8, device="cuda")
    back = spread(N, k, ld)
    m.ddit_mx4_quantize(u, ld, N, k, codes, scales)
    m.ddit_mx4_dequantize(codes, scales, N, k, back, ld)
    torch.cuda.synchronize()
    want_c, want_s = encode64(u.cpu())
    assert torch.equal(codes.cpu(), want_c) and torch.equal(scales.cpu(), want_s)
    assert torch.equal(back.double(), decode64(codes, scales, k))
    wc, ws, W64 = _weights(m, n, k, g)
    ld_out = (1 << 25) - 8
    out = spread(N, n, ld_out) if N * ld_out * 2 > 1 << 31 else torch.full((N, n), -7.0, dtype=torch.bfloat16, device="cuda")
    ld_out = out.stride(0)
    y, e = _product(u, W64, k)
    work = torch.empty(m.ddit_linear_mx4_workspace_bytes(N, n, k), dtype=torch.uint8, device="cuda")
    m.ddit_linear_mx4_fwd(0, u, ld, wc, ws, None, N, n, k, out, ld_out, work)
    torch.cuda.synchronize()
    assert ((out.double() - y).abs() <= e + 2.0 ** -8 * (y.abs() + e)).all()
    x = torch.randn(N, n, device="cuda", generator=g)
    x_out = torch.empty_like(x)
    out.fill_(-7.0)
    m.ddit_linear_mx4_fwd(2, u, ld, wc, ws, None, N, n, k, out, ld_out, work, resid=x, resid_out=x_out)
    torch.cuda.synchronize()
    y = x.double() + y
    e = e + 2 * U * (y.abs() + (y - x).abs())
    assert ((x_out.double() - y).abs() <= e).all() and ((out.double() - y).abs() <= e + 2.0 ** -8 * (y.abs() + e)).all()


def test_a_long_output_of_a_linear(m):
    """bf16 outputs of 2.3 GB, an fp32 stream of 4.6 GB, updated in place."""
    N, n, k = 140003, 8192, 40
    g = torch.Generator(device="cuda").manual_seed(4)
    u = torch.randn(N, k, device="cuda", generator=g).bfloat16()
    wc, ws, W64 = _weights(m, n, k, g)
    out = torch.empty((N, n), dtype=torch.bfloat16, device="cuda")
    work = torch.empty(m.ddit_linear_mx4_workspace_bytes(N, n, k), dtype=torch.uint8, device="cuda")
    at = torch.cat((some_rows(N, 2 * n), some_rows(N, 4 * n))).unique()
    y, e = _product(u[at], W64, k)
    m.ddit_linear_mx4_fwd(0, u, k, wc, ws, None, N, n, k, out, n, work)
    torch.cuda.synchronize()
    assert ((out[at].double() - y).abs() <= e + 2.0 ** -8 * (y.abs() + e)).all()
    x = torch.empty((N, n), device="cuda").normal_(0.0, 3.0, generator=g)
    before = x[at].double()
    assert m.ddit_linear_mx4_form(2, N, n, k) == (256, 256)
    m.ddit_linear_mx4_fwd(2, u, k, wc, ws, None, N, n, k, out, n, work, resid=x, resid_out=x)
    torch.cuda.synchronize()
    y, e = before + y, e + 2 * U * (y.abs() + (before + y).abs())
    assert ((x[at].double() - y).abs() <= e).all() and ((out[at].double() - y).abs() <= e + 2.0 ** -8 * (y.abs() + e)).all()


@pytest.mark.parametrize("tokens,states", [([3, 2, 595], [500, 40, 60]), ([20, 4, 1, 600], [300, 150, 0, 500]), ([5, 1], [300, 1400]), ([300] + [1] * 10, [300] + [5] * 10)])
@pytest.mark.parametrize("H,G,dh", [(4, 2, 72), (4, 4, 128)])
def test_attention_of_strided_rows(m, tokens, states, H, G, dh):
    ld = (1 << 22) - 8
    q_off, kv_off = offsets(tokens), offsets(states)
    R, K = q_off[-1], kv_off[-1]
    g = torch.Generator(device="cuda").manual_seed(5)
    draw = lambda rows, cols: torch.randn(rows, cols, device="cuda", generator=g)
    far = R * ld * 2 > 1 << 31
    q = spread(R, H * dh, ld, draw(R, H * dh)) if far else draw(R, H * dh).bfloat16()
    o = spread(R, H * dh, ld) if far else torch.empty_like(q)
    k, v = spread(K, G * dh, ld, draw(K, G * dh)), spread(K, G * dh, ld, draw(K, G * dh))
    lse = torch.empty((R, H), device="cuda")
    qo, ko = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (q_off, kv_off))
    work = torch.empty(m.ddit_cross_attn_packed_workspace_bytes(len(tokens), R, K, H, dh) or 256, dtype=torch.uint8, device="cuda")
    m.ddit_cross_attn_packed_fwd(q, q.stride(0), qo, k, v, ld, ko, None, len(tokens), R, K, H, G, dh, dh ** -0.5, o, o.stride(0), lse, work)
    torch.cuda.synchronize()
    ro, eo, rl, el = cross_reference(q, k, v, q_off, kv_off, None, H, G, dh, dh ** -0.5)
    assert ((o.double() - ro).abs() <= eo).all()
    none = rl == -math.inf
    assert torch.equal(lse == -math.inf, none) and ((lse.double() - rl).abs()[~none] <= el[~none]).all()
