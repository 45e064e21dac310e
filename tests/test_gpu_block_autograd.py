"""What the feed-forward block's autograd ops do for the engine around them."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ops():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    from paper_2609_14339_amd import block
    return block


def make(H=64, F=96, rows=20, dtype=torch.float32):
    g = torch.Generator().manual_seed(3)
    mk = lambda *s, k=1.0: (torch.randn(*s, generator=g) * k).to(dtype).cuda().requires_grad_()
    return dict(x=mk(rows, H), gamma=mk(H), beta=mk(H), W1=mk(F, H, k=1 / math.sqrt(H)), b1=mk(F),
                W2=mk(H, F, k=1 / math.sqrt(F)), b2=mk(H))


def outputs(ops, p):
    return {"layer_norm": lambda: ops.layer_norm(p["x"], p["gamma"], p["beta"]),
            "linear": lambda: ops.linear(p["x"], p["W1"], p["b1"], act="silu"),
            "mlp_block": lambda: ops.mlp_block(**p)}


@pytest.mark.parametrize("name", ["layer_norm", "linear", "mlp_block"])
def test_second_derivatives_raise(ops, name):
    """A penalty on a gradient beside an ordinary loss: an error, not a sum that lacks the penalty."""
    p = make()
    out = outputs(ops, p)[name]()
    (g,) = torch.autograd.grad(out.square().sum(), p["x"], create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable|differentiate twice"):
        (p["x"].sum() + g.square().sum()).backward()
