"""Packed cross-attention where scale q.k is far from zero, up to values that leave fp32.

Queries and keys are small whole numbers, so the scores are exact and any two differ by nothing or by at least one.  From a scale of 200 on
a state that is not among the best of a query has a weight of at most exp(-200): less than 2^-280.  So o is the mean of v over the best, n of
them, and lse = scale best + log n.

Tolerance.  The best states' weights are equal; they are off from the same power of two by at most 2^-12 (half a step of a reference of 4096,
where the kernel leaves it), which stays below half a bf16 step of the weights, in the sums of weights though not in their rounded form:
2^-11.  The sums of n terms add n 2^-24, the output's rounding 2^-8.  lse: the product, the sum and the logarithm's three operations are each
off by at most one unit of 2^-24 of |lse| + log n, the reference by another: 8 units; a value past fp32 is an infinity."""
import math

import pytest
import torch

from test_gpu_cross_packed import U, offsets, run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


def whole(g, low, high, *shape):
    return torch.randint(low, high + 1, shape, generator=g, device="cuda").float()


def check(q, k, v, q_off, kv_off, mask, H, G, dh, scale, o, lse):
    for b in range(len(q_off) - 1):
        rows = slice(q_off[b], q_off[b + 1])
        keys = torch.arange(kv_off[b], kv_off[b + 1], device="cuda")
        if mask is not None:
            keys = keys[mask[keys] != 0]
        if not len(keys):
            assert (o[rows] == 0).all() and (lse[rows] == -math.inf).all()
            continue
        for h in range(H):
            g = h // (H // G)
            s = q[rows, h * dh:(h + 1) * dh].double() @ k[keys, g * dh:(g + 1) * dh].double().t().contiguous()
            vd = v[keys, g * dh:(g + 1) * dh].double()
            best = s.amax(1)
            hit = (s == best[:, None]).double()
            n = hit.sum(1)
            want, size = hit @ vd / n[:, None], hit @ vd.abs() / n[:, None]
            got = o[rows, h * dh:(h + 1) * dh].double()
            assert ((got - want).abs() <= (2.0 ** -11 + n[:, None] * U) * size + 2.0 ** -8 * want.abs()).all(), (b, h)
            value = scale * best + torch.log(n)
            far = value.abs() >= 3.4028235e38
            assert torch.equal(lse[rows, h][far].double(), torch.sign(value[far]) * math.inf)
            assert ((lse[rows, h].double() - value).abs()[~far] <= (8 * U * (value.abs() + torch.log(n)))[~far]).all(), (b, h)


# few queries (a wavefront alone), keys in parts, keys resident, streamed, and three wavefronts a SIMD
FORMS = [([5, 1, 40], [65, 300, 7], 4, 2, 72), ([3, 2], [2000, 1500], 4, 2, 128), ([300, 0, 131], [300, 9, 0], 4, 4, 64), ([400, 90], [700, 30], 4, 4, 96),
         ([5000, 3400], [300, 400], 16, 16, 72)]


@pytest.mark.parametrize("tokens,states,H,G,dh", FORMS)
@pytest.mark.parametrize("scale", [200.0, 1e5, 2.0 ** 33, 1e12, 1e30, 1e37, 9e37])
@pytest.mark.parametrize("sign", [1, -1])
def test_far_scores(m, tokens, states, H, G, dh, scale, sign):
    """sign -1: every score is negative, so the best one is far below zero too."""
    g = torch.Generator(device="cuda").manual_seed(len(tokens) + dh)
    q_off, kv_off = offsets(tokens), offsets(states)
    q = (sign * whole(g, 1, 3, q_off[-1], H * dh)).bfloat16()
    kv = torch.randn(kv_off[-1], 2 * G * dh, generator=g, device="cuda")
    kv[:, :G * dh] = whole(g, 0, 3, kv_off[-1], G * dh)
    kv[:, 0:G * dh:dh] += 1          # no score is zero
    kv = kv.bfloat16()
    k, v = kv[:, :G * dh], kv[:, G * dh:]
    mask = (torch.rand(kv_off[-1], generator=g, device="cuda") > 0.3).to(torch.uint8)
    for use in (None, mask):
        o, lse = run(m, q, k, v, q_off, kv_off, use, H, G, dh, scale, H * dh, 2 * G * dh)
        check(q, k, v, q_off, kv_off, use, H, G, dh, scale, o, lse)


def test_flat_scores_of_any_size_weigh_alike(m):
    """All states alike: the mean of v, however far the common score is."""
    H, dh = 2, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    for R, K in ((7, 90), (4, 3000), (200, 300), (200, 800)):
        q, k = torch.ones(R, H * dh, device="cuda").bfloat16(), torch.ones(K, H * dh, device="cuda").bfloat16()
        v = torch.randn(K, H * dh, generator=g, device="cuda").bfloat16()
        for scale in (1e3, 1e9, 1e20, 1e37):
            o, lse = run(m, q, k, v, [0, R], [0, K], None, H, H, dh, scale, H * dh, H * dh)
            check(q, k, v, [0, R], [0, K], None, H, H, dh, scale, o, lse)


def test_one_query_without_weight_beside_far_ones(m):
    """In the first tiles one query's scores are -inf, its neighbours' are far from zero: neither disturbs the other."""
    H, dh, K, scale = 1, 64, 300, 1e8
    g = torch.Generator(device="cuda").manual_seed(6)
    for R in (5, 200):
        q, k = whole(g, 1, 3, R, dh), whole(g, 0, 3, K, dh)
        q[:, 0] = 0
        q[3, 0] = -4
        k[:, 0] = 0
        k[:128, 0] = 2.0 ** 127       # times -4: past fp32
        v = torch.randn(K, dh, generator=g, device="cuda").bfloat16()
        q, k = q.bfloat16(), k.bfloat16()
        o, lse = run(m, q, k, v, [0, R], [0, K], None, H, H, dh, scale, dh, dh)
        check(q, k, v, [0, R], [0, K], None, H, H, dh, scale, o, lse)
