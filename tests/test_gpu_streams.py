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
    key = pk.make_key(1, 0, 0, 0, 1, ROWS, H)
    K = pk.ac_keep_count(H, 0.1)
    vals, idx = pk.ac_mask_pack(x, K, key)
    row_ptr, bits = pk.ac_bern_mask(ROWS, H, 0.1, key)
    held = pk.ac_bern_pack(x, row_ptr, bits)[0]
    U, V, d = randn(ROWS, 8, seed=8, dtype=torch.float32), randn(H, 8, seed=9, dtype=torch.float32), torch.ones(8).cuda()
    tall = randn(H, ROWS, seed=10)

    def batched(s, tall, U, d, V, out, ws):
        pk.sc_correct_batched([dict(G=tall.t(), prior=(U, d, V), out=out, ws=ws)], 8, 0.3, stream=s)
        return out

    return {
        "ac_mask_pack": (lambda s, x: pk.ac_mask_pack(x, K, key, stream=s), [x]),
        "ac_unpack_scatter": (lambda s, v, i: pk.ac_unpack_scatter(v, H, key, 2.0, i, stream=s), [vals, idx]),
        "ac_mask_pack_batched": (lambda s, x: pk.ac_mask_pack_batched(x[None], K, key, stream=s), [x]),
        "ac_unpack_scatter_batched": (lambda s, v: pk.ac_unpack_scatter_batched(v[None], H, key, stream=s), [vals]),
        "ac_bern_mask": (lambda s: pk.ac_bern_mask(ROWS, H, 0.1, key, stream=s), []),
        "ac_bern_pack": (lambda s, x, r, b: pk.ac_bern_pack(x, r, b, stream=s), [x, row_ptr, bits]),
        "ac_bern_unpack": (lambda s, v, r, b: pk.ac_bern_unpack(v, H, r, b, stream=s), [held, row_ptr, bits]),
        "sc_build_prior": (lambda s, g, M: pk.sc_build_prior(g, M, 8, 0.0, 1e-3, 8, 2, stream=s),
                           [x, torch.zeros(ROWS, H).cuda()]),
        "sc_correct": (lambda s, t, *p: pk.sc_correct(t.t(), *p, 0.3, stream=s), [tall, U, d, V]),
        "sc_correct_batched": (batched, [tall, U, d, V, torch.empty_like(x), pk.workspace(ROWS, H, 8, 0, BF16)]),
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
         "lin_backward_input", "lin_backward_weight", "ac_mask_pack", "ac_unpack_scatter", "ac_mask_pack_batched",
         "ac_unpack_scatter_batched", "ac_bern_mask", "ac_bern_pack", "ac_bern_unpack", "sc_build_prior", "sc_correct",
         "sc_correct_batched"]


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
def test_results_and_inputs_that_are_dropped_at_once(pk, square, name):
    fn, inputs = calls(pk)[name]
    want = [t.clone() for t in flat(fn(None, *inputs))]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    busy(side, square)
    copies = [t.clone() for t in inputs]
    # a batched call's items are the caller's to keep, but for what it had to copy
    keep = copies[1:] if name == "sc_correct_batched" else None
    side.wait_stream(torch.cuda.current_stream())
    got = flat(fn(side, *copies))
    fn(side, *copies)                            # its results go at once
    sizes = [t.numel() * t.element_size() for t in (*copies, *want)]
    del copies
    other = [torch.empty(n, dtype=torch.uint8, device="cuda").fill_(7) for n in sizes for _ in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (keep is None or len(keep) == 5)
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


def test_compressor_outputs(pk, square):
    from paper_2609_14339_amd.powersgd import PowerSGDState
    g = randn(ROWS, H, seed=1)
    states = [PowerSGDState([(ROWS, H)], 8.0, BF16, g.device, seed=3) for _ in range(2)]
    want = states[0].step([g])[0].clone()
    torch.cuda.synchronize()
    held = blocks([want])
    busy(torch.cuda.current_stream(), square)
    for t in held:
        t.fill_(255)
    del held, t
    got = states[1].step([g], stream=torch.cuda.Stream())[0]
    torch.cuda.synchronize()
    assert torch.equal(got, want)
