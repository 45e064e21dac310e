"""Coded gated products whose pre-activations go through the workspace in runs of rows: every row of every run."""
import pytest
import torch

from test_gpu_glu import F32, check_forward, randn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    yield pk
    torch.cuda.empty_cache()


# two and more runs, the last of them short; inputs that are read where they are, at odd strides, and copied first
@pytest.mark.parametrize("dtype,rows,n_in,F,pad", [(F32, 40003, 24, 1030, 0), (F32, 70001, 33, 600, 3), (F32, 1 << 20, 33, 40, 1),
                                                   (F32, (1 << 20) + 5, 64, 40, 0), (F32, 20000, 300, 4100, 8)])
def test_forward(pk, dtype, rows, n_in, F, pad):
    plan = pk.glu_product_plan(pk.GLU_FORWARD, rows, n_in, F, dtype, True)
    assert plan.whole == 0 and 4 * plan.cut * plan.pieces * plan.tile_rows * plan.tile_cols > 256 << 20
    check_forward(pk, dtype, rows, n_in, F, "silu", pad=pad)


@pytest.mark.parametrize("n_in", [24, 27])
def test_runs_are_calls_of_their_rows(pk, n_in):
    """One step of the sum: a row's result is the same in a call of some rows alone, and in a graph."""
    rows, F = 40003, 1030
    x, W, b = randn(rows, n_in, dtype=F32, seed=1), randn(2 * F, n_in, dtype=F32, seed=2), randn(2 * F, dtype=F32, seed=3)
    h, pair = pk.glu_forward(x, W, b, keep="q8")
    for at in (0, 19000, 20000, 39800):
        some, kept = pk.glu_forward(x[at:at + 203], W, b, keep="q8")
        assert torch.equal(some, h[at:at + 203])
        for p, q in zip(kept, pair):
            assert torch.equal(p.codes, q.codes[at:at + 203]) and torch.equal(p.scales, q.scales[at:at + 203])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held, kept = pk.glu_forward(x, W, b, keep="q8")
    for i in range(3):
        x.copy_(torch.randn(rows, n_in, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        h, pair = pk.glu_forward(x, W, b, keep="q8")
        assert torch.equal(held, h) and all(torch.equal(a, b) for p, q in zip(kept, pair) for a, b in zip(p, q))


def test_a_workspace_of_the_stated_size(pk):
    rows, n_in, F = 40003, 24, 1030
    x, W = randn(rows, n_in, dtype=F32, seed=1), randn(2 * F, n_in, dtype=F32, seed=2)
    need = pk.glu_workspace_size(pk.GLU_FORWARD, rows, n_in, F, F32, True)
    ws = torch.full((need + 4096,), 77, dtype=torch.uint8, device="cuda")
    h, pair = pk.glu_forward(x, W, keep="q8", ws=ws[:need])
    assert (ws[need:] == 77).all()
    want, other = pk.glu_forward(x, W, keep="q8")
    assert torch.equal(h, want) and all(torch.equal(a, b) for p, q in zip(pair, other) for a, b in zip(p, q))
    with pytest.raises(pk.AcscError, match="needed"):
        pk.glu_forward(x, W, keep="q8", ws=ws[:need - 256])
