"""Gradients of the pass between two blocks that are wanted one by one: each as all of them together give it, and what is
not wanted is not formed."""
import pytest
import torch

from test_gpu_drop import kept, make
from test_gpu_gated_block import F32, branch, grads64, params, rel, rms
from test_gpu_join import EPS, SCALE, tensors

pytestmark = pytest.mark.gpu
NAMES = ("post", "gate", "pre")


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


@pytest.mark.parametrize("H", [130, 3000, 9001])
def test_of_the_call(pk, H):
    rows = 60
    t = tensors(rows, H, F32, 0)
    j = pk.join_forward(t["r"], t["b"], t["post"], t["gate"], t["pre"], SCALE, make(pk, rows, H, 0.1, 3), EPS)
    call = lambda **kw: pk.join_backward(t["dout"], t["dy"], j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"],
                                         SCALE, make(pk, rows, H, 0.1, 3), **kw)
    want = call()
    for names in ((), ("post",), ("gate",), ("pre",), ("post", "pre")):
        for dr in (True, False):
            d = call(weights=names, want_dr=dr)
            for name, a, b in zip(("dr", "db", "dpost", "dgate", "dpre"), d, want):
                asked = dr if name == "dr" else name == "db" or name[1:] in names
                assert torch.equal(a, b) if asked else a is None, name
    with pytest.raises(pk.AcscError, match="dr is given"):
        call(dr=torch.empty_like(t["dout"]), want_dr=False)
    with pytest.raises(pk.AcscError, match="dpost is given"):
        call(weights=("gate",), dpost=torch.empty(H, device="cuda"))
    with pytest.raises(pk.AcscError, match="weights"):
        call(weights=("gamma",))


@pytest.mark.parametrize("wanted", ["r", "b", *NAMES])
@pytest.mark.parametrize("used", ["out", "y", "both"])
def test_of_the_op(pk, wanted, used):
    from paper_2609_14339_amd.block import join
    rows, H = 40, 200
    g = torch.Generator().manual_seed(3)
    every = {k: torch.randn(rows, H, generator=g).cuda() for k in ("r", "b")}
    every.update({k: torch.randn(H, generator=g).cuda() for k in NAMES})
    ups = [torch.randn(rows, H, generator=g).cuda() for _ in range(2)]
    drop = make(pk, rows, H, 0.1)

    def grads(names):
        p = {k: v.clone().requires_grad_(k in names) for k, v in every.items()}
        outs = join(**p, scale=SCALE, drop=drop)
        pick = [i for i in range(2) if used in ("both", ("out", "y")[i])]
        return dict(zip(names, torch.autograd.grad([outs[i] for i in pick], [p[k] for k in names], [ups[i] for i in pick],
                                                   allow_unused=True)))
    got, want = grads([wanted])[wanted], grads(list(every))[wanted]
    if wanted == "pre" and used == "out":
        assert got is None and want is None
    else:
        assert torch.equal(got, want)


@pytest.mark.parametrize("x_wants", [True, False])
def test_a_block_of_scale_one(pk, x_wants):
    """The stream's gradient is then the result's own, and is not written again."""
    from paper_2609_14339_amd.block import glu_block
    rows, H, F = 50, 192, 130
    p = params(H, F, F32, 4)
    x = torch.randn(rows, H, generator=torch.Generator().manual_seed(5)).cuda().requires_grad_(x_wants)
    g = torch.randn(rows, H, generator=torch.Generator().manual_seed(6)).cuda()
    m, up = kept(rows, H, 0.2, 5)
    factor = (m.double() * float(up)).cuda()
    out = glu_block(x, **p, checkpoint=False, drop=make(pk, rows, H, 0.2, 5))
    got = torch.autograd.grad(out, [*p.values()] + ([x] if x_wants else []), g.clone())
    ref, want = grads64(lambda x, p: x + factor * p["gate"] * rms(branch(rms(x, p["gamma"]), p, "silu"), p["post"]), x, p, g)
    assert rel(out, ref) <= 1e-6
    for name, a, b in zip([*p, "x"], got, (*want[1:], want[0])):
        assert rel(a, b) <= 1e-5, name
