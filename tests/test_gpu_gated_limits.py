"""The gated block's calls on tensors of more than 2^31 elements and on more rows than a grid has workgroups across: the
last rows against 64-bit references, and the whole against the same call on its end alone."""
import math

import pytest
import torch

from test_gpu_drop import kept, make
from test_gpu_glu import act_pair
from test_gpu_join import EPS, SCALE, TOL, near, ref_backward, ref_forward

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    yield pk
    torch.cuda.empty_cache()


def gauss(rows, H, dtype, seed):
    return torch.randn(rows, H, generator=torch.Generator("cuda").manual_seed(seed), device="cuda", dtype=dtype)


@pytest.mark.parametrize("rows,H", [(70001, 32000), (1200003, 1100), (5000003, 64)])
def test_join(pk, rows, H):
    """More than 2^31 elements in wide rows; more than 2^20 workgroups of a row, and of four."""
    t = dict(r=gauss(rows, H, BF16, 1), b=gauss(rows, H, BF16, 2), dout=gauss(rows, H, BF16, 3), dy=gauss(rows, H, BF16, 4),
             **{k: (torch.randn(H, device="cuda") * 0.2 + 1).bfloat16() for k in ("post", "gate", "pre")})
    drop = make(pk, rows, H, 0.1, 3)
    m, up = kept(rows, H, 0.1, 3, first=rows - 3, count=3)
    factor = (m.double() * float(up)).cuda()
    j = pk.join_forward(t["r"], t["b"], t["post"], t["gate"], t["pre"], SCALE, drop, EPS)
    end = {k: v[-3:] if v.dim() == 2 else v for k, v in t.items()}
    ref = ref_forward(end, True, True, True, factor)
    near(j.out[-3:], ref["out"], TOL[BF16], ref["size"])
    near(j.y[-3:], ref["y"], TOL[BF16], ref["size_y"])
    d = pk.join_backward(t["dout"], t["dy"], j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE, drop,
                         dr=t["dout"])
    want, size = ref_backward({**end, "dout": gauss(rows, H, BF16, 3)[-3:]}, j.out[-3:], end["b"], j.rstd_post[-3:], j.rstd_pre[-3:],
                              True, True, True, factor)
    near(d.dr[-3:], want["dr"], TOL[BF16], size["dr"])
    near(d.db[-3:], want["db"], TOL[BF16], size["db"])
    # sums of unit normal terms: standard deviation sqrt(rows), far from it were rows lost or taken twice
    for v in (d.dpost, d.dgate, d.dpre):
        assert torch.isfinite(v).all() and v.abs().max() < 20 * rows ** 0.5


@pytest.mark.parametrize("keep", ["z", "q8"])
@pytest.mark.parametrize("rows,n_in,F", [(70001, 8, 16000), (3000001, 16, 8)])
def test_glu(pk, rows, n_in, F, keep):
    x, W = gauss(rows, n_in, BF16, 1), gauss(2 * F, n_in, BF16, 2) / math.sqrt(n_in)
    h, kept_ = pk.glu_forward(x, W, None, keep=keep)
    # the end alone, at which every row is its own
    eh, ek = pk.glu_forward(x[-300:], W, None, keep=keep)
    z = x[-300:].double() @ W.double().t()
    want = act_pair(z[:, :F], "silu")[0] * z[:, F:]
    # both roundings are of bf16; sums of n_in products differ by their order
    near(h[-300:], want, TOL[BF16])
    near(eh, want, TOL[BF16])
    if keep == "z":
        near(kept_[-300:], z, TOL[BF16])
        end = kept_[-300:]
    else:
        for i, q in enumerate(kept_):
            v = q.codes[-300:].double() * q.scales[-300:].double().repeat_interleave(128, 1)[:, :F]
            near(v, z[:, i * F:(i + 1) * F], 2e-2)
        end = tuple(pk.Q8(q.codes[-300:], q.scales[-300:]) for q in kept_)
    dy, W2 = gauss(rows, n_in, BF16, 3), gauss(n_in, F, BF16, 4)
    dz, hidden, dbias = pk.glu_backward_input(dy, W2, kept_, hidden=True, bias=True)
    edz, eh2, _ = pk.glu_backward_input(dy[-300:], W2, end, hidden=True, bias=True)
    near(dz[-300:], edz.double(), 2 * TOL[BF16])
    near(hidden[-300:], eh2.double(), 2 * TOL[BF16])
    # against the sums of the rounded dz, whose roundings add up as their squares do
    for half in (0, 1):
        part = dz[:, half * F:(half + 1) * F]
        s = torch.zeros(F, dtype=torch.float64, device="cuda")
        size = torch.zeros_like(s)
        for at in range(0, rows, 1 << 16):
            v = part[at:at + (1 << 16)].double()
            s += v.sum(0)
            size += v.square().sum(0)
        got = dbias[half * F:(half + 1) * F].double()
        assert ((got - s).abs() <= 8 * 2.0 ** -8 * size.sqrt() + 2.0 ** -24 * 300 * size.sqrt() * rows ** 0.5).all()
