"""The feed-forward block between two boundaries: its parts as autograd ops,
the whole block from 8-bit checkpoints, and its weight gradients through the
corrector."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def params(H, F, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    mk = lambda *s, k=1.0, b=0.0: (torch.randn(*s, generator=g) * k + b).to(dtype).cuda().requires_grad_()
    return dict(gamma=mk(H, k=0.1, b=1.0), beta=mk(H, k=0.1), W1=mk(F, H, k=1 / math.sqrt(H)), b1=mk(F, k=0.1),
                W2=mk(H, F, k=1 / math.sqrt(F)), b2=mk(H, k=0.1))


def reference(x, p, act):
    """The block in 64 bits under torch's own autograd."""
    F = torch.nn.functional
    h = F.layer_norm(x, (x.shape[-1],), p["gamma"], p["beta"], 1e-5)
    z = h @ p["W1"].t() + p["b1"]
    a = {"gelu": lambda t: 0.5 * t * torch.erfc(-t / math.sqrt(2)), "relu": torch.relu,
         "silu": lambda t: t * torch.sigmoid(t), "none": lambda t: t}[act](z)
    return x + a @ p["W2"].t() + p["b2"]


def rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


# fp32 and whole tensors: chains of fp32 sums, far below 1e-5.  8-bit: a value is off by at most half a step, a / 254
# of its group's largest; for normal values that is 3.5 / 254 / sqrt 3 = 0.8% of their scale.  It enters the gradients
# once through act' (second derivative at most 0.8) and the norm's input, once through each weight gradient's operand:
# under 2% in all.  bf16 adds roundings of 2^-9 at five places.
@pytest.mark.parametrize("act", ["gelu", "silu", "relu", "none"])
@pytest.mark.parametrize("dtype,checkpoint,tol", [(torch.float32, False, 1e-5), (torch.float32, True, 2e-2),
                                                  (torch.bfloat16, True, 3e-2)])
def test_block_gradients(pk, act, dtype, checkpoint, tol):
    from paper_2609_14339_amd.block import mlp_block
    if act == "relu" and dtype != torch.float32:
        pytest.skip("relu' at a rounded zero crossing is compared in fp32")
    B, S, H, F = 3, 43, 192, 400
    p = params(H, F, dtype)
    x = torch.randn(B, S, H, generator=torch.Generator().manual_seed(9)).to(dtype).cuda().requires_grad_()
    g = torch.randn(B, S, H, generator=torch.Generator().manual_seed(10)).to(dtype).cuda()
    out = mlp_block(x, **p, act=act, checkpoint=checkpoint)
    got = torch.autograd.grad(out, [x, *p.values()], g)
    x64 = x.detach().double().requires_grad_()
    p64 = {k: v.detach().double().requires_grad_() for k, v in p.items()}
    ref = reference(x64, p64, act)
    want = torch.autograd.grad(ref, [x64, *p64.values()], g.double())
    assert rel(out, ref.detach()) <= (1e-6 if dtype == torch.float32 else 6e-3)
    for name, a, b in zip(["x", *p], got, want):
        # a relu unit whose code crosses zero flips its gradient whole: about 1% of them, 10% of the norm
        t = 0.15 if act == "relu" and checkpoint else tol
        assert a.dtype == dtype and rel(a, b) <= t, name


def test_parts_as_ops_of_their_own(pk):
    from paper_2609_14339_amd.block import layer_norm, linear
    H, F = 96, 160
    p = params(H, F, torch.float32, seed=4)
    x = torch.randn(2, 17, H, device="cuda", requires_grad=True)
    h = layer_norm(x, p["gamma"], p["beta"])
    a = linear(h, p["W1"], p["b1"], act="silu")
    out = linear(a, p["W2"], p["b2"], residual=x)
    got = torch.autograd.grad(out.sum(), [x, *p.values()])          # an expanded gradient
    x64 = x.detach().double().requires_grad_()
    p64 = {k: v.detach().double().requires_grad_() for k, v in p.items()}
    want = torch.autograd.grad(reference(x64, p64, "silu").sum(), [x64, *p64.values()])
    for a, b in zip(got, want):
        assert rel(a, b) <= 1e-5


def test_what_a_block_keeps(pk):
    """Beside its parameters: 1.03 bytes a value of the input and of the pre-activation, and two numbers a row."""
    from paper_2609_14339_amd.block import mlp_block
    rows, H, F = 256, 1024, 4096
    p = params(H, F, torch.bfloat16, seed=1)
    x = torch.randn(rows, H, device="cuda").bfloat16().requires_grad_()
    kept = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: kept.append(t) or t, lambda t: t):
        mlp_block(x, **p)
    own = {t.data_ptr() for t in p.values()}
    size = sum(t.numel() * t.element_size() for t in kept if t.data_ptr() not in own)
    assert size == rows * (H + F) * (1 + 4 / 128) + 8 * rows


def test_stage_step_masks_block_and_corrector(pk):
    """A stage's step as a program runs it: the masked boundary, the block, the boundary's gradient, and the weight
    gradients corrected with an anchor prior."""
    from paper_2609_14339_amd.autograd import boundary_key, masked_boundary
    from paper_2609_14339_amd.block import mlp_block
    from paper_2609_14339_amd.prior import AnchorPrior
    B, S, H, F = 2, 64, 256, 512
    p = params(H, F, torch.bfloat16, seed=2)
    h = torch.randn(B, S, H, generator=torch.Generator().manual_seed(3)).bfloat16().cuda().requires_grad_()
    key = boundary_key(1, 0, 0, 0, h)
    x = masked_boundary(h, 0.1, key)
    out = mlp_block(x, **p)
    target = torch.randn(B, S, H, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    loss = (out - target).float().square().mean()
    gh, gW1, gW2 = torch.autograd.grad(loss, [h, p["W1"], p["W2"]])
    assert (gh[x == 0] == 0).all() and torch.isfinite(gh).all()
    prior = AnchorPrior([(F, H), (H, F)], 8, 0.9, 1e-3, 8, 2, dtype=torch.bfloat16)
    prior.arrive([gW1, gW2])
    out = prior.correct([gW1, gW2], 0.3)
    for c, g in zip(out, (gW1, gW2)):
        assert c.shape == g.shape and torch.isfinite(c).all()
        # the correction does not grow a gradient
        assert c.float().norm() <= 1.01 * g.float().norm()
