"""Cross-attention of packed requests against float64: lengths from nothing to thousands on both sides, masks that leave nothing,
infinities and NaN where nobody looks, strides, grouped heads, keys in parts.

Tolerance.  A score is a sum of dh products, off by at most (dh + 8) 2^-24 scale |q|.|k| =: d (its largest over the keys), and the exponent
by 4 2^-24 of the score's size, which d covers; so a weight is off by a factor of 1 + 2 d, and by half a bf16 step, 2^-8, for P V.  With
A = sum p |v| / sum p:  |o error| <= (2^-8 + 4 d + 80 2^-24) A, and 2^-8 of o for its own rounding.  The logarithm: 2 d + 80 2^-24."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


def offsets(lengths, first=0):
    o = [first]
    for n in lengths:
        o.append(o[-1] + n)
    return o


def reference(q, k, v, q_off, kv_off, mask, H, G, dh, scale):
    """float64 -> o, its tolerance, lse, its tolerance; NaN in the rows of no sequence"""
    R = q.shape[0]
    o = torch.full((R, H, dh), math.nan, dtype=torch.float64, device=q.device)
    lse = torch.full((R, H), math.nan, dtype=torch.float64, device=q.device)
    eo, el = torch.zeros_like(o), torch.zeros_like(lse)
    for b in range(len(q_off) - 1):
        rows = slice(q_off[b], q_off[b + 1])
        if rows.start == rows.stop:
            continue
        keys = torch.arange(kv_off[b], kv_off[b + 1], device=q.device)
        if mask is not None:
            keys = keys[mask[keys] != 0]
        if not len(keys):
            o[rows], lse[rows] = 0, -math.inf
            continue
        for h in range(H):
            g = h // (H // G)
            qd = q[rows, h * dh:(h + 1) * dh].double()
            kd, vd = (t[keys, g * dh:(g + 1) * dh].double().contiguous() for t in (k, v))
            s = scale * (qd @ kd.t().contiguous())
            d = ((dh + 8) * U * scale * (qd.abs() @ kd.abs().t().contiguous())).amax(1, keepdim=True)
            lse[rows, h] = torch.logsumexp(s, 1)
            p = torch.exp(s - lse[rows, h][:, None])
            o[rows, h] = p @ vd
            eo[rows, h] = (2.0 ** -8 + 4 * d + 80 * U) * (p @ vd.abs()) + 2.0 ** -8 * o[rows, h].abs()
            el[rows, h] = 2 * d[:, 0] + 80 * U + U * lse[rows, h].abs()
    return o.view(R, H * dh), eo.view(R, H * dh), lse, el


def run(m, q, k, v, q_off, kv_off, mask, H, G, dh, scale, ld_q, ld_kv, ld_o=None, want_lse=True, R=None, K=None):
    R, K, B = R or q.shape[0], K if K is not None else k.shape[0], len(q_off) - 1
    ld_o = ld_o or H * dh
    o = torch.full((max(R, 1), ld_o), -7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((max(R, 1), H), -7.0, device="cuda") if want_lse else None
    ws = torch.full((m.ddit_cross_attn_packed_workspace_bytes(B, R, K, H, dh),), 0xFF, dtype=torch.uint8, device="cuda")
    qo, ko = (torch.tensor(t, dtype=torch.int32, device="cuda") for t in (q_off, kv_off))
    m.ddit_cross_attn_packed_fwd(q, ld_q, qo, k, v, ld_kv, ko, mask, B, R, K, H, G, dh, scale, o, ld_o, lse, ws if ws.numel() else None)
    torch.cuda.synchronize()
    return o, lse


def inputs(R, K, H, G, dh, seed, gain=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(*s, device="cuda", generator=g)
    return (gain * draw(max(R, 1), H * dh)).bfloat16(), draw(max(K, 1), 2 * G * dh).bfloat16(), g


def check(m, tokens, states, H, G, dh, masked=False, seed=1, gain=1.0, scale=None, first=0, want_lse=True):
    q_off, kv_off = offsets(tokens, first), offsets(states, first)
    R, K = q_off[-1] + first, kv_off[-1] + first
    q, kv, g = inputs(R, K, H, G, dh, seed, gain)
    k, v = kv[:, :G * dh], kv[:, G * dh:]
    mask = (torch.rand(max(K, 1), device="cuda", generator=g) > 0.3).to(torch.uint8) * 3 if masked else None
    scale = scale or dh ** -0.5
    o, lse = run(m, q, k, v, q_off, kv_off, mask, H, G, dh, scale, H * dh, 2 * G * dh, want_lse=want_lse, K=K)
    ro, eo, rl, el = reference(q, k, v, q_off, kv_off, mask, H, G, dh, scale)
    own = ~rl[:, 0].isnan()
    assert (o[~own] == -7).all()
    assert ((o[own].double() - ro[own]).abs() <= eo[own]).all(), float(((o[own].double() - ro[own]).abs() - eo[own]).max())
    if want_lse:
        assert (lse[~own] == -7).all()
        none = rl == -math.inf
        assert torch.equal(lse == -math.inf, none)
        fine = own[:, None] & ~none
        assert ((lse.double() - rl).abs()[fine] <= el[fine]).all()
    return o, lse


@pytest.mark.parametrize("dh", [8, 40, 64, 72, 80, 88, 96, 104, 128])
def test_head_dims(m, dh):
    check(m, [130, 1, 31], [65, 300, 7], 4, 4, dh, seed=dh)
    check(m, [5, 1], [700, 130], 4, 2, dh, seed=dh, masked=True)


@pytest.mark.parametrize("tokens,states", [
    ([1], [1]), ([1], [64]), ([1], [65]), ([32], [63]), ([33], [128]), ([127, 129], [64, 1]), ([128], [129]), ([0, 5, 0], [3, 3, 3]), ([5, 5, 5], [0, 3, 0]),
    ([7], [0]), ([0, 0, 1], [0, 0, 0]), ([600, 1, 77], [120, 300, 0]), ([3, 2, 0, 4], [4096, 1, 5, 2500]), ([2, 1], [5000, 0]), ([1] * 70, list(range(70))),
    ([64] * 3, [1000, 10, 2000]), ([65] * 3, [1000, 10, 2000]), ([0] * 130 + [3] + [0] * 70 + [40], [5] * 202), ([4000], [300]), ([1500, 200], [1024, 2048])])
@pytest.mark.parametrize("masked", [False, True])
def test_lengths(m, tokens, states, masked):
    check(m, tokens, states, 3, 3, 72, masked, seed=len(tokens) + states[0])


@pytest.mark.parametrize("H,G", [(1, 1), (16, 16), (16, 4), (8, 1), (6, 2)])
def test_grouped_heads(m, H, G):
    check(m, [50, 200], [90, 33], H, G, 64, seed=H)
    check(m, [4, 9], [900, 1500], H, G, 128, seed=H, want_lse=False)


def test_rows_of_no_sequence_stay(m):
    check(m, [40, 9], [70, 80], 2, 2, 72, first=5)
    check(m, [3, 2], [1500, 800], 2, 2, 72, first=5, masked=True)


@pytest.mark.parametrize("gain,scale", [(30.0, None), (1.0, 5.0), (0.0, None), (1.0, 1e-6), (1.0, 1e-39)])
def test_peaked_and_flat(m, gain, scale):
    for tokens, states in [([100, 30], [200, 333]), ([2, 3], [2000, 1500])]:
        check(m, tokens, states, 2, 2, 72, gain=gain, scale=scale, seed=7)


def test_growing_scores_move_the_maximum(m):
    """Keys in ascending order of their score: every tile beats the running maximum."""
    H, dh, K = 2, 64, 1024
    for R in (3, 200):
        q, kv, _ = inputs(R, K, H, H, dh, 3)
        q = q.abs()
        k = torch.linspace(-4, 4, K, device="cuda")[:, None].expand(K, H * dh).bfloat16().contiguous()
        v = kv[:, :H * dh].contiguous()
        o, lse = run(m, q, k, v, [0, R], [0, K], None, H, H, dh, 1.0, H * dh, H * dh)
        ro, eo, rl, el = reference(q, k, v, [0, R], [0, K], None, H, H, dh, 1.0)
        assert ((o.double() - ro).abs() <= eo).all() and ((lse.double() - rl).abs() <= el).all()


@pytest.mark.parametrize("tokens,states", [([40, 140, 5], [100, 130, 64]), ([3, 5, 1], [1500, 2000, 900])])
def test_what_a_mask_takes_out_may_hold_anything(m, tokens, states):
    H, G, dh = 4, 2, 72
    q_off, kv_off = offsets(tokens), offsets(states)
    R, K = q_off[-1], kv_off[-1]
    q, kv, g = inputs(R, K, H, G, dh, 5)
    mask = (torch.rand(K, device="cuda", generator=g) > 0.5).to(torch.uint8)
    mask[kv_off[1]:kv_off[2]] = 0                       # nothing left of the second request
    k, v = kv[:, :G * dh], kv[:, G * dh:]
    a = run(m, q, k, v, q_off, kv_off, mask, H, G, dh, 0.1, H * dh, 2 * G * dh)
    out = (mask == 0).nonzero()[:, 0]
    for i, bad in enumerate((math.inf, -math.inf, math.nan, 3.3e38)):
        kv[out[i::4]] = bad
    b = run(m, q, k, v, q_off, kv_off, mask, H, G, dh, 0.1, H * dh, 2 * G * dh)
    assert torch.equal(a[0].view(torch.int16), b[0].view(torch.int16)) and torch.equal(a[1], b[1])
    rows = slice(q_off[1], q_off[2])
    assert (b[0][rows] == 0).all() and (b[1][rows] == -math.inf).all() and b[0].isfinite().all()
    # a request's neighbours may hold anything too
    mask.fill_(1)
    kv.copy_(inputs(R, K, H, G, dh, 5)[1])
    a = run(m, q, k, v, q_off, kv_off, None, H, G, dh, 0.1, H * dh, 2 * G * dh)
    kv[kv_off[1]:kv_off[2]] = math.nan
    q[q_off[1]:q_off[2]] = math.inf
    b = run(m, q, k, v, q_off, kv_off, None, H, G, dh, 0.1, H * dh, 2 * G * dh)
    for r in (slice(0, q_off[1]), slice(q_off[2], R)):
        assert torch.equal(a[0][r].view(torch.int16), b[0][r].view(torch.int16)) and torch.equal(a[1][r], b[1][r])
    assert b[0][rows].isnan().all() and b[1][rows].isnan().all()


def test_scores_of_minus_infinity_and_a_bad_query(m):
    """Weights of exactly zero in whole tiles, and a query that is NaN: alone."""
    H, dh, K = 1, 64, 300
    for R in (4, 100):
        q, kv, _ = inputs(R, K, H, H, dh, 9)
        q[:, 0] = 1.0
        k, v = kv[:, :dh].contiguous(), kv[:, dh:].contiguous()
        k[:128, 0] = -math.inf
        o, lse = run(m, q, k, v, [0, R], [0, K], None, H, H, dh, 0.125, dh, dh)
        ro, eo, rl, el = reference(q, k[128:], v[128:], [0, R], [0, K - 128], None, H, H, dh, 0.125)
        assert ((o.double() - ro).abs() <= eo).all() and ((lse.double() - rl).abs() <= el).all()
        q[2, 5] = math.nan
        o2, lse2 = run(m, q, k, v, [0, R], [0, K], None, H, H, dh, 0.125, dh, dh)
        assert o2[2].isnan().all() and lse2[2].isnan().all()
        keep = torch.arange(R, device="cuda") != 2
        assert torch.equal(o2[keep].view(torch.int16), o[keep].view(torch.int16)) and torch.equal(lse2[keep], lse[keep])


@pytest.mark.parametrize("tokens,states", [([40, 140], [100, 130]), ([3, 5], [1500, 900])])
def test_strides(m, tokens, states):
    H, G, dh = 4, 2, 72
    q_off, kv_off = offsets(tokens), offsets(states)
    R, K = q_off[-1], kv_off[-1]
    q, kv, _ = inputs(R, K, H, G, dh, 11)
    k, v = kv[:, :G * dh], kv[:, G * dh:]
    a = run(m, q, k, v, q_off, kv_off, None, H, G, dh, 0.1, H * dh, 2 * G * dh)
    wide_q = torch.full((R, 3 * H * dh + 8), math.nan, dtype=torch.bfloat16, device="cuda")
    wide_q[:, 8:8 + H * dh] = q
    wide_k = torch.full((K, 5 * G * dh), math.nan, dtype=torch.bfloat16, device="cuda")
    wide_k[:, G * dh:2 * G * dh], wide_k[:, 3 * G * dh:4 * G * dh] = k, v
    b = run(m, wide_q[:, 8:], wide_k[:, G * dh:], wide_k[:, 3 * G * dh:], q_off, kv_off, None, H, G, dh, 0.1, 3 * H * dh + 8, 5 * G * dh, ld_o=H * dh + 16)
    assert torch.equal(a[0].view(torch.int16), b[0][:, :H * dh].contiguous().view(torch.int16)) and torch.equal(a[1], b[1])
    assert (b[0][:, H * dh:] == -7).all()


def test_offsets_outside_the_arrays_are_cut_off(m):
    H, dh = 2, 64
    q, kv, _ = inputs(100, 200, H, H, dh, 13)
    k, v = kv[:, :H * dh], kv[:, H * dh:]
    a = run(m, q, k, v, [0, 40, 100], [0, 90, 200], None, H, H, dh, 0.1, H * dh, 2 * H * dh)
    b = run(m, q, k, v, [-5, 40, 1 << 30], [-9, 90, 2147483647], None, H, H, dh, 0.1, H * dh, 2 * H * dh)
    assert torch.equal(a[0].view(torch.int16), b[0].view(torch.int16)) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("R,K", [(400, 700), (12, 3000)])
def test_a_captured_call_serves_other_lengths(m, R, K):
    H, G, dh, B = 4, 2, 72, 3
    q, kv, g = inputs(R, K, H, G, dh, 17)
    k, v = kv[:, :G * dh], kv[:, G * dh:]
    mask = torch.ones(K, dtype=torch.uint8, device="cuda")
    qo, ko = (torch.zeros(B + 1, dtype=torch.int32, device="cuda") for _ in range(2))
    o, lse = torch.empty((R, H * dh), dtype=torch.bfloat16, device="cuda"), torch.empty((R, H), device="cuda")
    ws = torch.empty(m.ddit_cross_attn_packed_workspace_bytes(B, R, K, H, dh) or 256, dtype=torch.uint8, device="cuda")
    call = lambda: m.ddit_cross_attn_packed_fwd(q, H * dh, qo, k, v, 2 * G * dh, ko, mask, B, R, K, H, G, dh, 0.1, o, H * dh, lse, ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for i, (a, b) in enumerate([((0, R // 2, R // 2, R), (0, K // 3, K // 2, K)), ((0, 1, 2, R - 3), (7, 7, 100, K)), ((0, R, R, R), (0, K, K, K))]):
        qo.copy_(torch.tensor(a)), ko.copy_(torch.tensor(b))
        mask.copy_(torch.rand(K, generator=torch.Generator().manual_seed(i)) > 0.2)
        o.fill_(-7.0), lse.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        want = run(m, q, k, v, list(a), list(b), mask, H, G, dh, 0.1, H * dh, 2 * G * dh)
        assert torch.equal(o.view(torch.int16), want[0].view(torch.int16)) and torch.equal(lse, want[1])
        ro, eo, rl, el = reference(q, k, v, a, b, mask, H, G, dh, 0.1)
        own = ~rl[:, 0].isnan()
        assert ((o[own].double() - ro[own]).abs() <= eo[own]).all()


def test_no_states_and_no_queries_at_all(m):
    H, dh = 2, 64
    q, kv, _ = inputs(9, 20, H, H, dh, 1)
    o, lse = run(m, q, kv[:0, :H * dh], kv[:0, H * dh:], [0, 4, 9], [0, 0, 0], None, H, H, dh, 0.1, H * dh, 2 * H * dh, K=0)
    assert (o == 0).all() and (lse == -math.inf).all()
    off = torch.zeros(2, dtype=torch.int32, device="cuda")
    m.ddit_cross_attn_packed_fwd(q[:0], H * dh, off, kv, kv, 2 * H * dh, off, None, 1, 0, 20, H, H, dh, 0.1, o[:0], H * dh, lse[:0], None)
    torch.cuda.synchronize()


@pytest.mark.parametrize("H,G,dh", [(16, 16, 72), (16, 16, 64), (32, 16, 96), (16, 16, 128)])
def test_many_rows(m, H, G, dh):
    """From 512 row tiles of 256 on heads of up to 96 features take three wavefronts a SIMD: resident and streamed keys, a ragged end."""
    tokens = [5000, 301, 0, 3100] if G == H else [2500, 301, 0, 1600]
    check(m, tokens, [300, 77, 5, 700], H, G, dh, seed=dh)
    check(m, tokens, [64, 0, 9, 257], H, G, dh, masked=True, seed=dh + 1)
