"""The gated feed-forward block: its parts as autograd ops, blocks in a row joined by one pass, the whole block from
8-bit checkpoints, and its weight gradients through the corrector."""
import math

import pytest
import torch

from test_gpu_drop import kept, make

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS = 1e-5


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def params(H, F, dtype, seed=0):
    g = torch.Generator().manual_seed(seed)
    mk = lambda *s, k=1.0, b=0.0: (torch.randn(*s, generator=g) * k + b).to(dtype).cuda().requires_grad_()
    return dict(gamma=mk(H, k=0.1, b=1.0), W=mk(2 * F, H, k=1 / math.sqrt(H)), bias=mk(2 * F, k=0.1),
                W2=mk(H, F, k=1 / math.sqrt(F)), bias2=mk(H, k=0.1), post=mk(H, k=0.1, b=1.0), gate=mk(H, k=0.1, b=0.4))


def rms(x, w):
    return x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w


def act64(t, act):
    return {"gelu": lambda t: 0.5 * t * torch.erfc(-t / math.sqrt(2)), "relu": torch.relu,
            "silu": lambda t: t * torch.sigmoid(t), "none": lambda t: t}[act](t)


def branch(y, p, act):
    z = y @ p["W"].t() + p["bias"]
    F = z.shape[-1] // 2
    return (act64(z[..., :F], act) * z[..., F:]) @ p["W2"].t() + p["bias2"]


def rel(a, b):
    a, b = a.detach().double(), b.detach().double()
    return float((a - b).norm() / b.norm())


def grads64(f, x, p, g):
    x64 = x.detach().double().requires_grad_()
    p64 = {k: v.detach().double().requires_grad_() for k, v in p.items()}
    ref = f(x64, p64)
    return ref.detach(), torch.autograd.grad(ref, [x64, *p64.values()], g.double())


# fp32 and whole tensors: chains of fp32 sums, far below 1e-5.  8-bit: a value is off by at most half a step, a / 254 of
# its group's largest; for normal values 3.5 / 254 / sqrt 3 = 0.8% of their scale.  It enters the gradients through the
# gate's value and slope, the up value, the norms' inputs: five such at most in one product of terms, under 4% in all.
# bf16 adds roundings of 2^-8 at seven places.
@pytest.mark.parametrize("form", ["plain", "whole"])
@pytest.mark.parametrize("act", ["silu", "gelu", "none"])
@pytest.mark.parametrize("dtype,checkpoint,tol", [(F32, False, 1e-5), (F32, True, 4e-2), (BF16, True, 5e-2)])
def test_block_gradients(pk, act, dtype, checkpoint, tol, form):
    from paper_2609_14339_amd.block import glu_block
    B, S, H, F = 3, 43, 192, 400
    p = params(H, F, dtype)
    x = torch.randn(B, S, H, generator=torch.Generator().manual_seed(9)).to(dtype).cuda().requires_grad_()
    g = torch.randn(B, S, H, generator=torch.Generator().manual_seed(10)).to(dtype).cuda()
    if form == "plain":
        p.pop("post"), p.pop("gate")
        out = glu_block(x, **p, act=act, checkpoint=checkpoint)
        f = lambda x, p: x + branch(rms(x, p["gamma"]), p, act)
    else:
        m, up = kept(B * S, H, 0.2, 5, B=B)
        factor = (m.double() * float(up)).cuda().view(B, S, H)
        out = glu_block(x, **p, act=act, checkpoint=checkpoint, scale=0.5, drop=make(pk, B * S, H, 0.2, 5, B=B))
        f = lambda x, p: 0.5 * x + factor * p["gate"] * rms(branch(rms(x, p["gamma"]), p, act), p["post"])
    got = torch.autograd.grad(out, [x, *p.values()], g)
    ref, want = grads64(f, x, p, g)
    assert rel(out, ref) <= (1e-6 if dtype == F32 else 1.5e-2)
    for name, a, b in zip(["x", *p], got, want):
        assert a.dtype == dtype and a.shape == b.shape and rel(a, b) <= tol, name


def test_blocks_in_a_row_joined_in_one_pass(pk):
    """Two blocks from their parts: norm, gated product, down projection, and the pass between the blocks, which takes
    the norm after the first, its gate, dropout and residual, and the norm before the second."""
    from paper_2609_14339_amd.block import dropout, glu, join, linear, rms_norm
    rows, H, F = 70, 160, 96
    p, p2 = params(H, F, F32, 1), params(H, F, F32, 2)
    x = torch.randn(2, 35, H, device="cuda", requires_grad=True)
    d1, d2 = make(pk, rows, H, 0.1, 0, B=2), make(pk, rows, H, 0.1, 1, B=2)
    f1, f2 = ((kept(rows, H, 0.1, s, B=2)[0].double() * 65536 / 58982).cuda().view(2, 35, H) for s in (0, 1))

    def part(y, p):
        return linear(glu(y, p["W"], p["bias"]), p["W2"], p["bias2"])
    r, y = join(x, part(rms_norm(x, p["gamma"], EPS), p), p["post"], p["gate"], p2["gamma"], 0.75, d1, EPS)
    out = dropout(part(y, p2), d2, residual=r)
    every = {**{"a_" + k: v for k, v in p.items()}, **{"b_" + k: v for k, v in p2.items() if k not in ("post", "gate")}}
    g = torch.randn(2, 35, H, device="cuda")
    got = torch.autograd.grad(out, [x, *every.values()], g)

    def ref(x, q):
        a, b = ({k[2:]: v for k, v in q.items() if k.startswith(s)} for s in ("a_", "b_"))
        r = 0.75 * x + f1 * a["gate"] * rms(branch(rms(x, a["gamma"]), a, "silu"), a["post"])
        return r + f2 * branch(rms(r, b["gamma"]), b, "silu")
    want_out, want = grads64(ref, x, every, g)
    assert rel(out, want_out) <= 1e-6
    for name, a, b in zip(["x", *every], got, want):
        assert rel(a, b) <= 1e-5, name


def test_parts_alone_and_unused_results(pk):
    from paper_2609_14339_amd.block import dropout, join, rms_norm
    H = 130
    x = torch.randn(40, H, device="cuda", requires_grad=True)
    b = torch.randn(40, H, device="cuda", requires_grad=True)
    w = torch.ones(H, device="cuda", requires_grad=True)
    # only the stream, or only the next block's input, is used
    for k in (0, 1):
        parts = join(x, b, post=w, pre=w, checkpoint=False)
        got = torch.autograd.grad(parts[k].sum(), [x, b, w])
        x64, b64, w64 = (t.detach().double().requires_grad_() for t in (x, b, w))
        r = x64 + rms(b64, w64)
        want = torch.autograd.grad((r, rms(r, w64))[k].sum(), [x64, b64, w64])
        for u, v in zip(got, want):
            assert rel(u, v) <= 1e-5
    # no gains, no gradients wanted of them; an expanded gradient
    y = rms_norm(x)
    got, = torch.autograd.grad(y.sum(), [x])
    x64 = x.detach().double().requires_grad_()
    want, = torch.autograd.grad(rms(x64, 1.0).sum(), [x64])
    assert (got.double() - want).norm() <= 1e-5 * (1 / rms(x64, 1.0).detach() * x64.detach()).norm()
    # dropout's gradient goes through the same mask
    d = make(pk, 40, H, 0.5, 7)
    out = dropout(x, d)
    got, = torch.autograd.grad(out.sum(), [x])
    assert torch.equal(got, torch.where(out != 0, got, 0.0)) and ((got == 0) == (out == 0)).all()


@pytest.mark.parametrize("name", ["glu", "join", "dropout", "rms_norm", "glu_block"])
def test_second_derivatives_raise(pk, name):
    """A penalty on a gradient beside an ordinary loss: an error, not a sum that lacks the penalty."""
    from paper_2609_14339_amd import block
    p = params(64, 32, F32, 5)
    x = torch.randn(8, 64, device="cuda", requires_grad=True)
    out = {"glu": lambda: block.glu(x, p["W"], p["bias"]), "join": lambda: block.join(x, x, p["post"]),
           "dropout": lambda: block.dropout(x, make(pk, 8, 64, 0.1)), "rms_norm": lambda: block.rms_norm(x, p["gamma"]),
           "glu_block": lambda: block.glu_block(x, **p)}[name]()
    (g,) = torch.autograd.grad(out.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError, match="once_differentiable|differentiate twice"):
        (x.sum() + g.square().sum()).backward()


def test_what_a_block_keeps(pk):
    """Beside its parameters: 1.03 bytes a value of the input, both pre-activations and the branch, two numbers a row;
    and no mask."""
    from paper_2609_14339_amd.block import glu_block
    rows, H, F = 256, 1024, 2048
    p = params(H, F, BF16, seed=1)
    x = torch.randn(rows, H, device="cuda").bfloat16().requires_grad_()
    saved = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: saved.append(t) or t, lambda t: t):
        glu_block(x, **p, drop=make(pk, rows, H, 0.1))
    own = {t.data_ptr() for t in p.values()}
    size = sum(t.numel() * t.element_size() for t in saved if t.data_ptr() not in own)
    assert size == rows * (2 * H + 2 * F) * (1 + 4 / 128) + 8 * rows


def test_stage_step_masks_block_and_corrector(pk):
    """A stage's step as a program runs it: the masked boundary, the block with its dropout keyed by the same step, the
    boundary's gradient, and the weight gradients corrected with an anchor prior."""
    from paper_2609_14339_amd.autograd import boundary_key, masked_boundary
    from paper_2609_14339_amd.block import glu_block
    from paper_2609_14339_amd.prior import AnchorPrior
    B, S, H, F = 2, 64, 256, 512
    p = params(H, F, BF16, seed=2)
    h = torch.randn(B, S, H, generator=torch.Generator().manual_seed(3)).bfloat16().cuda().requires_grad_()
    key = boundary_key(1, 0, 0, 0, h)
    x = masked_boundary(h, 0.1, key)
    out = glu_block(x, **p, drop=pk.Drop(0.1, key))
    target = torch.randn(B, S, H, generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    loss = (out - target).float().square().mean()
    gh, gW, gW2 = torch.autograd.grad(loss, [h, p["W"], p["W2"]])
    assert (gh[x == 0] == 0).all() and torch.isfinite(gh).all()
    prior = AnchorPrior([(2 * F, H), (H, F)], 8, 0.9, 1e-3, 8, 2, dtype=BF16)
    prior.arrive([gW, gW2])
    for c, g in zip(prior.correct([gW, gW2], 0.3), (gW, gW2)):
        assert c.shape == g.shape and torch.isfinite(c).all()
        assert c.float().norm() <= 1.01 * g.float().norm()      # the correction does not grow a gradient


def test_a_step_in_a_graph(pk):
    """Forward and backward of a block captured and replayed (no eager graph of the same leaves is alive then)."""
    from paper_2609_14339_amd.block import glu_block
    rows, H, F = 96, 128, 192
    p = params(H, F, BF16, 3)
    x = torch.randn(rows, H, device="cuda").bfloat16().requires_grad_()
    g = torch.randn(rows, H, device="cuda").bfloat16()
    d = make(pk, rows, H, 0.1)
    leaves = [x, *p.values()]
    step = lambda: [(o := glu_block(x, **p, drop=d)).detach(), *torch.autograd.grad(o, leaves, g)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(3):
        with torch.no_grad():
            x.copy_(torch.randn(rows, H, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, step()):
            assert torch.equal(a, b)


def test_checkpoints_of_the_parts_between_blocks(pk):
    """join keeps in 8 bits what its backward pass reads and nothing else, and takes its gradients from that."""
    from paper_2609_14339_amd.block import join
    rows, H = 64, 512
    g = torch.Generator().manual_seed(3)
    mk = lambda *s: torch.randn(*s, generator=g).cuda().requires_grad_()
    r, b, gains = mk(rows, H), mk(rows, H), [mk(H) for _ in range(3)]
    for post, gate, pre in ((0, 0, 0), (1, 0, 0), (0, 1, 1), (1, 1, 1), (0, 0, 1)):
        kw = dict(post=gains[0] if post else None, gate=gains[1] if gate else None, pre=gains[2] if pre else None)
        saved = []
        with torch.autograd.graph.saved_tensors_hooks(lambda t: saved.append(t) or t, lambda t: t):
            outs = join(r, b, **kw, checkpoint=True)
        size = sum(t.numel() * t.element_size() for t in saved if all(t.data_ptr() != w.data_ptr() for w in gains))
        assert size == rows * H * (1 + 4 / 128) * (pre + (post or gate)) + 4 * rows * (post + pre)
        outs = outs if pre else (outs,)
        ups = [torch.randn(rows, H, generator=g).cuda() for _ in outs]
        wanted = [r, b, *(w for w in kw.values() if w is not None)]
        got = torch.autograd.grad(outs, wanted, ups)
        want = torch.autograd.grad(join(r, b, **kw) if pre else (join(r, b, **kw),), wanted, ups)
        for u, v in zip(got, want):      # values off by at most half a step: 0.8% of their scale, twice
            assert rel(u, v) <= 2e-2


@pytest.mark.parametrize("wanted", ["x", "gamma", "W", "bias", "W2", "bias2", "post", "gate"])
def test_only_one_gradient_wanted(pk, wanted):
    """Each gradient by itself is the one that all of them together give."""
    from paper_2609_14339_amd.block import glu_block
    p = {k: v.detach() for k, v in params(96, 64, F32, 6).items()}
    p["x"] = torch.randn(40, 96, generator=torch.Generator().manual_seed(1)).cuda()
    g, d = torch.randn(40, 96, generator=torch.Generator().manual_seed(2)).cuda(), make(pk, 40, 96, 0.1)
    every = {k: v.clone().requires_grad_() for k, v in p.items()}
    want = dict(zip(every, torch.autograd.grad(glu_block(**every, drop=d), list(every.values()), g)))
    one = {k: v.clone().requires_grad_(k == wanted) for k, v in p.items()}
    got, = torch.autograd.grad(glu_block(**one, drop=d), [one[wanted]], g)
    assert torch.equal(got, want[wanted])


@pytest.mark.parametrize("rows", [1, 50])
def test_evaluation_keeps_nothing(pk, rows):
    """Where no gradient is wanted the same results come without anything kept."""
    from paper_2609_14339_amd import block
    H, F = 256, 4096
    p = params(H, F, BF16, 7)
    x = torch.randn(rows, H, device="cuda").bfloat16()
    ops = {"glu_block": lambda: block.glu_block(x, **p), "glu": lambda: block.glu(x, p["W"], p["bias"], checkpoint=True),
           "join": lambda: block.join(x, x, p["post"], p["gate"], p["gamma"], checkpoint=True)[1],
           "rms_norm": lambda: block.rms_norm(x, p["gamma"], checkpoint=True)}
    for name, op in ops.items():
        want = op()
        assert want.requires_grad, name
        with torch.no_grad():
            got = op()
        # few tokens: with codes the pieces are added up in another kernel, in another order of fp32 sums
        assert not got.requires_grad and rel(got, want) <= 2.0 ** -8, name
        with torch.no_grad():
            assert torch.equal(op(), got)
