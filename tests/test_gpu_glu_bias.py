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
