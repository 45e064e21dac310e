"""Calls on a stream that is not the current one: their own memory, what they are given and what they return."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16
ROWS, H, F = 512, 1024, 1536


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def randn(*shape, seed, dtype=BF16):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def flat(out):
    if isinstance(out, torch.Tensor):
        return [out]
    return [t for o in out or () for t in flat(o)]


def calls(pk):
    """{name: (function of its inputs and a stream, inputs)}"""
    x, W, b = randn(ROWS, H, seed=1), randn(F, H, seed=2), randn(F, seed=3)
    dz, dy, z = randn(ROWS, F, seed=4), randn(ROWS, H, seed=5), randn(ROWS, H, seed=6)
    gamma = randn(H, seed=7)
    q = pk.q8_encode(x)
    _, mean, rstd, _ = pk.ln_forward(x)
    return {
        "q8_encode": (lambda s, x: pk.q8_encode(x, stream=s), [x]),
        "q8_decode": (lambda s, c, k: pk.q8_decode(pk.Q8(c, k), BF16, "silu", stream=s), list(q)),
        "ln_forward": (lambda s, x, g: pk.ln_forward(x, g, checkpoint=True, stream=s), [x, gamma]),
        "ln_recompute": (lambda s, x, m, r: pk.ln_recompute(x, m, r, stream=s), [x, mean, rstd]),
        "ln_backward": (lambda s, dy, c, k, m, r, g: pk.ln_backward(dy, pk.Q8(c, k), m, r, g, stream=s),
                        [dy, *q, mean, rstd, gamma]),
        "lin_forward": (lambda s, x, W, b: pk.lin_forward(x, W, b, "gelu", keep="q8", stream=s), [x, W, b]),
        "lin_backward_act": (lambda s, dy, z: pk.lin_backward_act(dy, z, "silu", stream=s), [dy, z]),
        "lin_backward_input": (lambda s, dz, W, z: pk.lin_backward_input(dz, W, "gelu", z, stream=s), [dz, W, z]),
        "lin_backward_weight": (lambda s, dz, z: pk.lin_backward_weight(dz, z, "gelu", stream=s), [dz, z]),
    }


NAMES = ["q8_encode", "q8_decode", "ln_forward", "ln_recompute", "ln_backward", "lin_forward", "lin_backward_act",
         "lin_backward_input", "lin_backward_weight"]


def busy(stream, a):
    """Some milliseconds of work."""
    with torch.cuda.stream(stream):
        for _ in range(8):
            torch.mm(a, a)


@pytest.fixture(scope="module")
def square():
    a = torch.zeros(8192, 8192, dtype=BF16, device="cuda")
    torch.mm(a, a)
    torch.cuda.synchronize()
    return a


def blocks(outs):
    """Tensors of every size that the call may allocate (its results, and workspaces up to 64 MB)."""
    sizes = {t.numel() * t.element_size() for t in outs} | {1 << k for k in range(9, 27)}
    return [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sorted(sizes) for _ in range(3)]


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_writes(pk, square, name):
    fn, inputs = calls(pk)[name]
    want = flat(fn(None, *inputs))
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
def test_results_and_inputs_that_are_dropped_at_once(pk, square, name):
    fn, inputs = calls(pk)[name]
    want = flat(fn(None, *inputs))
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


def test_results_used_and_dropped_on_the_current_stream(pk, square):
    """What a call returned stays whole while the current stream, which it was handed to, still reads it."""
    fn, inputs = calls(pk)["lin_forward"]
    want = flat(fn(None, *inputs))[0]
    torch.cuda.synchronize()
    side, here = torch.cuda.Stream(), torch.cuda.current_stream()
    y = flat(fn(side, *inputs))[0]
    here.wait_stream(side)
    busy(here, square)
    copy = y.clone()
    size = y.numel() * y.element_size()
    del y
    with torch.cuda.stream(side):
        other = [torch.empty(size, dtype=torch.uint8, device="cuda").fill_(7) for _ in range(4)]
    torch.cuda.synchronize()
    assert torch.equal(copy, want) and len(other) == 4


def test_the_current_stream_given_by_name(pk):
    fn, inputs = calls(pk)["lin_forward"]
    want, got = flat(fn(None, *inputs)), flat(fn(torch.cuda.current_stream(), *inputs))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
