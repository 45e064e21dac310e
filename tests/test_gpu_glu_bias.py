"""The bias gradient of the gated product from a given gradient of its result: sums of what dz is before its rounding."""
import math

import pytest
import torch

from test_gpu_glu import BF16, F32, U, act_pair, randn, within

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def pair_values(pk, kept, F):
    v = kept.double() if isinstance(kept, torch.Tensor) else torch.cat([pk.q8_decode(q, F32) for q in kept], 1).double()
    return v[:, :F], v[:, F:]


def sums64(dh, g, u, act, dtype):
    """The sums in 64 bits, and the bound of fp32 terms and of an fp32 sum of them in any order."""
    rows = dh.shape[0]
    a, slope = act_pair(g, act)
    ea = 4 * U * g.abs() + 2 * U * a.abs() + (1e-7 * g.abs() if dtype == BF16 else 0)
    es = 16 * U * (1 + g.abs()) + (2e-7 if dtype == BF16 else 0)
    want = torch.cat((dh * u * slope, dh * a), 1)
    term = torch.cat(((dh * u).abs() * es, dh.abs() * ea), 1)
    return want.sum(0), (term + U * (rows + 8) * want.abs()).sum(0)


@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_bias_gradient_of_the_autograd_op(pk, act, checkpoint):
    """One rounding to the bias's type: columns whose terms cancel show that no term was rounded before the sum."""
    from paper_2609_14339_amd import block
    rows, n_in, F = 300, 64, 500
    x, W = randn(rows, n_in, dtype=BF16, seed=1), randn(2 * F, n_in, dtype=BF16, seed=2, scale=1 / math.sqrt(n_in))
    bias = randn(2 * F, dtype=BF16, seed=3, scale=0.1).requires_grad_()
    dh = randn(rows, F, dtype=BF16, seed=4)
    got, = torch.autograd.grad(block.glu(x, W, bias, act, checkpoint), [bias], dh)
    g, u = pair_values(pk, pk.glu_forward(x, W, bias.detach(), act, keep="q8" if checkpoint else "z")[1], F)
    want, tol = sums64(dh.double(), g, u, act, BF16)
    assert got.dtype == BF16
    within(got, want, tol * (1 + 2.0 ** -8) + 2.0 ** -8 * want.abs())


# (rows, F): one row, one column, rows of one partial and of many, segments of 512 columns filled and not
SHAPES = [(1, 1), (1, 600), (15, 512), (17, 513), (64, 7), (300, 1030), (2001, 130), (40000, 24), (1100, 4100), (4097, 512)]


@pytest.mark.parametrize("kept_as", ["whole", "q8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,F", SHAPES)
def test_sums(pk, dtype, rows, F, kept_as):
    act, pad = ("silu", "gelu", "relu", "none")[(rows + F) % 4], (0, 8, 3)[rows % 3]
    z, dh = randn(rows, 2 * F, dtype=dtype, seed=rows + F, pad=pad), randn(rows, F, dtype=dtype, seed=rows + F + 1, pad=pad)
    kept = z if kept_as == "whole" else (pk.q8_encode(z[:, :F]), pk.q8_encode(z[:, F:]))
    dz0, h0 = pk.glu_backward_act(dh, kept, act, hidden=True)
    dz, h, db = pk.glu_backward_act_bias(dh, kept, act, hidden=True)
    assert torch.equal(dz, dz0) and torch.equal(h, h0)
    g, u = pair_values(pk, kept, F)
    want, tol = sums64(dh.double(), g, u, act, dtype)
    within(db, want, tol)
    dz2, none, db2 = pk.glu_backward_act_bias(dh, kept, act)
    assert none is None and torch.equal(dz2, dz) and torch.equal(db2, db)
    base = randn(2 * F, dtype=F32, seed=5)
    more = base.clone()
    pk.glu_backward_act_bias(dh, kept, act, dbias=more, accumulate=True)
    assert torch.equal(more, base + db)
    if kept_as == "whole":             # in the place of both inputs
        wide, at = torch.full((rows + 1, 2 * F + 3), 9.0, dtype=dtype, device="cuda"), dh.clone()
        wide[:rows, :2 * F] = z
        into = wide[:rows, :2 * F]
        assert torch.equal(pk.glu_backward_act_bias(at, into, act, dz=into, h=at)[2], db)
        assert torch.equal(into, dz) and torch.equal(at, h) and (wide[rows] == 9).all() and (wide[:, 2 * F:] == 9).all()


def test_no_rows_streams_graphs_and_workspaces(pk):
    e = torch.empty(0, 96, dtype=BF16, device="cuda")
    assert (pk.glu_backward_act_bias(e, torch.empty(0, 192, dtype=BF16, device="cuda"))[2] == 0).all()
    rows, F = 500, 700
    z, dh = randn(rows, 2 * F, dtype=BF16, seed=1), randn(rows, F, dtype=BF16, seed=2)
    want = pk.glu_backward_act_bias(dh, z, hidden=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = pk.glu_backward_act_bias(dh, z, hidden=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ws = torch.empty(pk.glu_bias_workspace_size(rows, F), dtype=torch.uint8, device="cuda")
    assert torch.equal(pk.glu_backward_act_bias(dh, z, ws=ws)[2], want[2])
    with pytest.raises(pk.AcscError, match="needed"):
        pk.glu_backward_act_bias(dh, z, ws=ws[:-1])
    with pytest.raises(pk.AcscError, match="accumulate"):
        pk.glu_backward_act_bias(dh, z, accumulate=True)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = pk.glu_backward_act_bias(dh, z, hidden=True)
    for _ in range(3):
        dh.copy_(torch.randn(rows, F, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, pk.glu_backward_act_bias(dh, z, hidden=True)))
