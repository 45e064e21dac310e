"""The gated block's calls on a stream that is not the current one: their own memory, what they are given and what they
return."""
import pytest
import torch

from test_gpu_streams import BF16, F, H, ROWS, blocks, busy, flat, randn, square  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def calls(pk):
    """{name: (function of its inputs and a stream, inputs)}"""
    x, W, bias = randn(ROWS, H, seed=1), randn(2 * F, H, seed=2), randn(2 * F, seed=3)
    dy, dh, z, W2 = randn(ROWS, H, seed=4), randn(ROWS, F, seed=5), randn(ROWS, 2 * F, seed=6), randn(H, F, seed=7)
    gains = [randn(H, seed=8 + i) for i in range(3)]
    drop = pk.Drop(0.1, pk.make_key(1, 0, 0, 0, 1, ROWS, H), 2)
    j = pk.join_forward(x, dy, *gains[:2], pre=gains[2], drop=drop, checkpoint=True)
    _, rstd, q = pk.rms_forward(x, gains[0], checkpoint=True)
    pair = [t for v in (pk.q8_encode(z[:, :F]), pk.q8_encode(z[:, F:])) for t in v]
    two = lambda a, b, c, d: (pk.Q8(a, b), pk.Q8(c, d))
    return {
        "drop_apply": (lambda s, x, r: pk.drop_apply(x, drop, r, stream=s), [x, dy]),
        "rms_forward": (lambda s, x, g: pk.rms_forward(x, g, checkpoint=True, stream=s), [x, gains[0]]),
        "rms_recompute": (lambda s, c, k, r, g: pk.rms_recompute(pk.Q8(c, k), r, g, stream=s), [*q, rstd, gains[0]]),
        "rms_backward": (lambda s, dy, x, r, g: pk.rms_backward(dy, x, r, g, stream=s), [dy, x, rstd, gains[0]]),
        "join_forward": (lambda s, r, b, p, g, n: pk.join_forward(r, b, p, g, n, drop=drop, checkpoint=True, stream=s),
                         [x, dy, *gains]),
        "join_backward": (lambda s, a, b, oc, ok, bc, bk, rp, rn, p, g, n: pk.join_backward(
            a, b, *two(oc, ok, bc, bk), rp, rn, p, g, n, drop=drop, stream=s),
            [x, dy, *j.q_out, *j.q_b, j.rstd_post, j.rstd_pre, *gains]),
        "glu_forward": (lambda s, x, W, b: pk.glu_forward(x, W, b, keep="q8", stream=s), [x, W, bias]),
        "glu_backward_act": (lambda s, dh, *q: pk.glu_backward_act(dh, two(*q), hidden=True, stream=s), [dh, *pair]),
        "glu_backward_input": (lambda s, dy, W, *q: pk.glu_backward_input(dy, W, two(*q), hidden=True, bias=True, stream=s),
                               [dy, W2, *pair]),
    }


NAMES = ["drop_apply", "rms_forward", "rms_recompute", "rms_backward", "join_forward", "join_backward", "glu_forward",
         "glu_backward_act", "glu_backward_input"]


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_writes(pk, square, name):  # noqa: F811
    fn, inputs = calls(pk)[name]
    want = [t.clone() for t in flat(fn(None, *inputs))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    held = blocks(want)
    torch.cuda.synchronize()
    busy(torch.cuda.current_stream(), square)
    for t in held:
        t.fill_(255)
    del held, t                                  # free, with the fills still to come
    got = flat(fn(side, *inputs))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(got) == len(want)


@pytest.mark.parametrize("name", NAMES)
def test_results_and_inputs_that_are_dropped_at_once(pk, square, name):  # noqa: F811
    fn, inputs = calls(pk)[name]
    want = [t.clone() for t in flat(fn(None, *inputs))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy(side, square)
    copies = [t.clone() for t in inputs]
    side.wait_stream(torch.cuda.current_stream())
    got = flat(fn(side, *copies))
    fn(side, *copies)                            # its results go at once
    sizes = [t.numel() * t.element_size() for t in (*copies, *want)]
    del copies
    other = [torch.empty(n, dtype=torch.uint8, device="cuda").fill_(7) for n in sizes for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(bool((t == 7).all()) for t in other)
