"""fp32 activations in the tails, where what is left of them is small: relative bounds."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


@pytest.mark.parametrize("rows", [2, 200])
def test_gelu_of_negative_values(pk, rows):
    """The argument z / sqrt 2 is rounded twice (3 U), which erfc magnifies by about z^2 + 1; erfc, the products and the
    exponential add a few units.  Down to -12, where Phi is 2e-33."""
    z = torch.linspace(-12, 6, 4001).cuda()
    z64 = z.double()
    phi = 0.5 * torch.erfc(-z64 / math.sqrt(2))
    density = torch.exp(-z64 * z64 / 2) / math.sqrt(2 * math.pi)
    units = (3 * (z64 * z64 + 1) + 16) * U
    x, W = torch.zeros(rows, 8, device="cuda"), torch.zeros(len(z), 8, device="cuda")
    y = pk.lin_forward(x, W, z, "gelu")[0].double()
    assert ((y - z64 * phi).abs() <= units * (z64 * phi).abs()).all()
    zz = z.expand(rows, -1).contiguous()
    slope = pk.lin_backward_act(torch.ones_like(zz), zz, "gelu").double()
    assert ((slope - (phi + z64 * density)).abs() <= units * (phi + z64.abs() * density)).all()


def test_gelu_of_negative_values_read_back(pk):
    z = torch.linspace(-12, -4, 33 * 128).view(33, 128).cuda()
    q = pk.q8_encode(z)
    v = pk.q8_decode(q, torch.float32).double()
    y = pk.q8_decode(q, torch.float32, act="gelu").double()
    want = 0.5 * v * torch.erfc(-v / math.sqrt(2))
    assert ((y - want).abs() <= (3 * (v * v + 1) + 16) * U * want.abs()).all()


@pytest.mark.parametrize("rows", [2, 200])
def test_silu_of_negative_values(pk, rows):
    """exp(-|z|) of an exact argument, a quotient and a product."""
    z = torch.linspace(-80, 6, 4001).cuda()
    z64 = z.double()
    s = torch.sigmoid(z64)
    x, W = torch.zeros(rows, 8, device="cuda"), torch.zeros(len(z), 8, device="cuda")
    y = pk.lin_forward(x, W, z, "silu")[0].double()
    assert ((y - z64 * s).abs() <= 16 * U * (z64 * s).abs()).all()
    zz = z.expand(rows, -1).contiguous()
    slope = pk.lin_backward_act(torch.ones_like(zz), zz, "silu").double()
    assert ((slope - s * (1 + z64 * (1 - s))).abs() <= 16 * U * s * (1 + z64.abs() * (1 - s))).all()
