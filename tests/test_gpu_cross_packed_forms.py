"""Every form of the packed cross-attention on head dims that fill its registers and that do not: a lone wavefront, eight with resident and
with streamed keys, a walk over several row tiles, parts of the keys.  The form that a case is meant for is asked for, so that a changed rule
cannot leave one untested.  Tolerances as in the module that holds the reference."""
import pytest
import torch

from test_gpu_cross_packed import check, inputs, offsets, run

pytestmark = pytest.mark.gpu
DIMS = [8, 40, 64, 72, 80, 88, 96, 104, 128]


@pytest.fixture(scope="module")
def m():
    import paper_2506_13497_amd as mod
    return mod


def form(m, tokens, states, H, G, dh):
    return m.ddit_cross_attn_packed_form(len(tokens), sum(tokens), sum(states), H, G, dh)


@pytest.mark.parametrize("dh", DIMS)
@pytest.mark.parametrize("G", [4, 2])
def test_eight_wavefronts(m, dh, G):
    tokens = [300, 1, 131]
    for states, masked in (([65, 300, 7], False), ([256, 257, 64], True), ([700, 0, 130], False), ([321, 320, 90], True)):
        assert form(m, tokens, states, 4, G, dh)[:2] == (8, 1)
        check(m, tokens, states, 4, G, dh, masked, seed=dh)


@pytest.mark.parametrize("dh", DIMS)
def test_a_lone_wavefront_in_parts(m, dh):
    assert form(m, [5, 1, 40], [1700, 130, 3], 4, 2, dh)[0] == 1 and form(m, [5, 1, 40], [1700, 130, 3], 4, 2, dh)[1] > 1
    check(m, [5, 1, 40], [1700, 130, 3], 4, 2, dh, seed=dh)
    check(m, [5, 1, 40], [1700, 130, 3], 4, 2, dh, True, seed=dh + 1)


@pytest.mark.parametrize("dh", [64, 72, 96, 128])
@pytest.mark.parametrize("states,masked", [([300], False), ([256], True), ([700], False), ([1], False), ([0], False)])
def test_several_row_tiles_of_eight_wavefronts(m, dh, states, masked):
    """One request of 6481 tokens: the queries of a wavefront's next row tile are asked for ahead of time, up to 96 features."""
    waves, parts, rows = form(m, [6481], states, 16, 16, dh)
    assert (waves, parts) == (8, 1) and rows >= 512
    check(m, [6481], states, 16, 16, dh, masked, seed=dh)


@pytest.mark.parametrize("dh", DIMS)
@pytest.mark.parametrize("states", [[700, 400], [1000, 100], [3996, 100]])
def test_eight_wavefronts_in_parts(m, dh, states):
    """Three parts: of up to four key tiles, which are resident, of five and six, and of 21, which are streamed."""
    assert form(m, [1500, 500], states, 8, 8, dh) == (8, 3, 256)
    check(m, [1500, 500], states, 8, 8, dh, masked=dh % 16 == 0, seed=dh)


@pytest.mark.parametrize("dh", [40, 72, 88])
def test_twelve_wavefronts_of_padded_heads(m, dh):
    tokens = [5000, 0, 3333]
    for states in ([300, 20, 65], [333, 20, 700]):
        assert form(m, tokens, states, 16, 16, dh)[:2] == (12, 1)
        check(m, tokens, states, 16, 16, dh, masked=dh == 72, seed=dh)


@pytest.mark.parametrize("tokens,states,H,G,dh", [([5, 40], [300, 7], 4, 2, 72), ([5, 1], [3000, 90], 4, 2, 128), ([300, 131], [700, 64], 4, 4, 96),
                                                  ([1500, 500], [4000, 96], 8, 8, 72), ([5000, 3400], [300, 77], 16, 16, 72)])
def test_the_same_bits_every_time(m, tokens, states, H, G, dh):
    q_off, kv_off = offsets(tokens), offsets(states)
    q, kv, _ = inputs(q_off[-1], kv_off[-1], H, G, dh, 3)
    call = lambda: run(m, q, kv[:, :G * dh], kv[:, G * dh:], q_off, kv_off, None, H, G, dh, dh ** -0.5, H * dh, 2 * G * dh)
    o, lse = call()
    for _ in range(3):
        a, b = call()
        assert torch.equal(a.view(torch.int16), o.view(torch.int16)) and torch.equal(b, lse)
