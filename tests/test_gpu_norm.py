"""Layer norm, forward and backward, against 64-bit references and
differences; from tensors and from 8-bit checkpoints."""
import pytest
import torch

pytestmark = pytest.mark.gpu
GROUP = 128
EPS = 1e-5
# bf16 outputs: one rounding, at most 2^-9 of each element.  fp32: sums of H terms in a tree of at most 3 + 32 + 10
# levels and a handful of operations on each element, of values of the row's scale.
BF16 = 2.0 ** -9 + 2e-5
F32 = 64 * 2.0 ** -24
TOL = {torch.bfloat16: BF16, torch.float32: F32}


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def near(got, want, tol):
    got, want = got.double().cpu(), want.double().cpu()
    assert torch.isfinite(got).all()
    d, n = (got - want).norm(), want.norm()
    assert d <= tol * n + 1e-30, f"{float(d / n):.3e} > {tol:.3e}"


def tensors(rows, H, dtype, pad, seed=0):
    g = torch.Generator().manual_seed(seed + H)
    mk = lambda *s: torch.randn(*s, generator=g).to(dtype).cuda()
    x = (torch.randn(rows, H + pad, generator=g) + 0.5).to(dtype).cuda()[:, :H]
    return x, mk(H), mk(H), mk(rows, H + pad)[:, :H], mk(rows, H + pad)[:, :H]


def ref_forward(x, gamma, beta):
    x = x.double()
    mu = x.mean(1, keepdim=True)
    rs = 1 / ((x - mu).square().mean(1, keepdim=True) + EPS).sqrt()
    return (x - mu) * rs * gamma.double() + beta.double(), mu[:, 0], rs[:, 0]


def ref_backward(dy, x, mu, rs, gamma, add):
    dy, x, mu, rs = dy.double(), x.double(), mu.double()[:, None], rs.double()[:, None]
    h = (x - mu) * rs
    g = dy * gamma.double()
    dx = rs * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
    return dx + (add.double() if add is not None else 0), (dy * h).sum(0), dy.sum(0)


SHAPES = [(1, 1, 0), (1, 64, 0), (2, 7, 0), (5, 500, 3), (129, 512, 0), (7, 1000, 8), (6, 1030, 5), (131, 2048, 0),
          (9, 2049, 0), (33, 4096, 0), (3, 5001, 1), (17, 8192, 0), (2, 12289, 0), (3, 28672, 0), (2, 32768, 0)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,H,pad", SHAPES)
def test_forward(pk, dtype, rows, H, pad):
    x, gamma, beta, _, _ = tensors(rows, H, dtype, pad)
    y, mu, rs, q = pk.ln_forward(x, gamma, beta, EPS, checkpoint=True)
    ry, rmu, rrs = ref_forward(x, gamma, beta)
    near(mu, rmu, F32)
    near(rs, rrs, F32)
    near(y, ry, TOL[dtype])
    want = pk.q8_encode(x)
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    y1, mu1, rs1, none = pk.ln_forward(x, gamma, beta, EPS)
    assert none is None and torch.equal(y1, y) and torch.equal(mu1, mu) and torch.equal(rs1, rs)
    # again, from the tensor (the same bits) and from the checkpoint (the formula on its values)
    assert torch.equal(pk.ln_recompute(x, mu, rs, gamma, beta, dtype), y)
    v = pk.q8_decode(q, torch.float32).double()
    near(pk.ln_recompute(q, mu, rs, gamma, beta, dtype),
         (v - mu.double()[:, None]) * rs.double()[:, None] * gamma.double() + beta.double(), TOL[dtype])
    # without weights
    near(pk.ln_forward(x, None, None, EPS)[0], ref_forward(x, torch.ones(H, device="cuda"), torch.zeros(H, device="cuda"))[0],
         TOL[dtype])


@pytest.mark.parametrize("kept", ["whole", "q8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,H,pad", SHAPES + [(3000, 256, 0), (2500, 4100, 4)])
def test_backward(pk, dtype, rows, H, pad, kept):
    x, gamma, beta, dy, add = tensors(rows, H, dtype, pad)
    _, mu, rs, q = pk.ln_forward(x, gamma, beta, EPS, checkpoint=True)
    src, value = (q, pk.q8_decode(q, torch.float32)) if kept == "q8" else (x, x)
    dx, dg, db = pk.ln_backward(dy, src, mu, rs, gamma, add=add)
    rdx, rdg, rdb = ref_backward(dy, value, mu, rs, gamma, add)
    near(dx, rdx, TOL[dtype])
    # column sums: at most `rows` additions and eight roundings on the way of each term
    h = (value.double() - mu.double()[:, None]) * rs.double()[:, None]
    for got, want, terms in ((dg, rdg, dy.double() * h), (db, rdb, dy.double())):
        assert ((got.double() - want).abs() <= 2.0 ** -24 * (rows + 8) * terms.abs().sum(0) + 1e-30).all()
    again = pk.ln_backward(dy, src, mu, rs, gamma, add=add)
    assert all(torch.equal(a, b) for a, b in zip(again, (dx, dg, db)))
    # no residual branch, no weights
    near(pk.ln_backward(dy, src, mu, rs)[0], ref_backward(dy, value, mu, rs, torch.ones(H, device="cuda"), None)[0],
         TOL[dtype] if H > 2 else 1.0)


def test_accumulates_and_works_in_place(pk):
    x, gamma, beta, dy, add = tensors(300, 1000, torch.bfloat16, 0)
    _, mu, rs, _ = pk.ln_forward(x, gamma, beta, EPS)
    dx, dg, db = pk.ln_backward(dy, x, mu, rs, gamma, add=add)
    sg, sb = torch.randn(1000, device="cuda"), torch.randn(1000, device="cuda")
    g2, b2 = sg.clone(), sb.clone()
    into = add.clone()
    pk.ln_backward(dy, x, mu, rs, gamma, add=into, dx=into, dgamma=g2, dbeta=b2, accumulate=True)
    assert torch.equal(into, dx) and torch.equal(g2, sg + dg) and torch.equal(b2, sb + db)
    into = dy.clone()
    pk.ln_backward(into, x, mu, rs, gamma, add=add, dx=into)
    assert torch.equal(into, dx)
    z = x.clone()
    want = pk.ln_forward(x, gamma, beta, EPS)[0]
    pk.ln_forward(z, gamma, beta, EPS, y=z)
    assert torch.equal(z, want)


def test_constant_and_masked_rows(pk):
    """A row that the mask left empty is constant: its variance is 0, its output beta."""
    x = torch.zeros(4, 640, device="cuda")
    x[1] = 3.0
    x[2, 5] = 20.0
    gamma, beta = torch.randn(640, device="cuda"), torch.randn(640, device="cuda")
    y, mu, rs, q = pk.ln_forward(x, gamma, beta, EPS, checkpoint=True)
    assert torch.equal(y[0], beta) and torch.equal(y[1], beta) and torch.equal(y[3], beta)
    ry, _, _ = ref_forward(x, gamma, beta)
    near(y, ry, F32)
    dy = torch.randn(4, 640, device="cuda")
    near(pk.ln_backward(dy, q, mu, rs, gamma)[0],
         ref_backward(dy, pk.q8_decode(q, torch.float32), mu, rs, gamma, None)[0], F32)


def test_a_non_finite_row_stays_alone(pk):
    x, gamma, beta, dy, add = tensors(70, 1500, torch.float32, 0)
    y0, mu0, rs0, _ = pk.ln_forward(x, gamma, beta, EPS)
    bad = x.clone()
    bad[13, 700] = float("nan")
    bad[40, 3] = float("inf")
    y, mu, rs, _ = pk.ln_forward(bad, gamma, beta, EPS)
    rows = [r for r in range(70) if r not in (13, 40)]
    assert torch.equal(y[rows], y0[rows]) and torch.isnan(y[13]).all() and torch.isnan(y[40]).any()
    dx = pk.ln_backward(dy, bad, mu, rs, gamma)[0]
    assert torch.equal(dx[rows], pk.ln_backward(dy, x, mu0, rs0, gamma)[0][rows])


def test_no_rows(pk):
    e = torch.empty(0, 96, device="cuda")
    g = torch.ones(96, device="cuda")
    y, mu, rs, q = pk.ln_forward(e, g, g, EPS, checkpoint=True)
    assert y.shape == (0, 96) and mu.shape == (0,)
    dx, dg, db = pk.ln_backward(e, e, mu, rs, g)
    assert dx.shape == (0, 96) and (dg == 0).all() and (db == 0).all()
    keep = torch.full((96,), 2.0, device="cuda")
    pk.ln_backward(e, q, mu, rs, g, dgamma=keep, dbeta=keep.clone(), accumulate=True)
    assert (keep == 2).all()


@pytest.mark.parametrize("H", [96, 3000])
def test_gradients_against_differences(pk, H):
    """Central differences of the fp32 forward pass along random directions:
    truncation h^2 / 6 of a third derivative of order 1, rounding 2^-24 |f| / h
    per output; h = 2^-7 leaves both under 1e-4 of the sums compared."""
    x, gamma, beta, dy, _ = tensors(8, H, torch.float32, 0)
    _, mu, rs, _ = pk.ln_forward(x, gamma, beta, EPS)
    dx, dg, db = pk.ln_backward(dy, x, mu, rs, gamma)
    f = lambda x, g, b: (pk.ln_forward(x, g, b, EPS)[0].double() * dy.double()).sum()
    h = 2.0 ** -7
    for which, grad in ((0, dx), (1, dg), (2, db)):
        d = torch.randn_like(grad)
        args = lambda s: [t + s * h * d if i == which else t for i, t in enumerate((x, gamma, beta))]
        diff = (f(*args(1)) - f(*args(-1))) / (2 * h)
        scale = float((grad.double() * d.double()).norm())
        assert abs(float(diff - (grad.double() * d.double()).sum())) <= 2e-3 * scale


@pytest.mark.parametrize("kept", ["whole", "q8"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_wide_rows_whose_sums_take_a_pass_of_their_own(pk, dtype, kept):
    """More than 16384 columns, enough rows for several slices of the column sums; dx in place of dy."""
    rows, H = 131, 16385 if dtype == torch.float32 else 20000
    x, gamma, beta, dy, add = tensors(rows, H, dtype, 0)
    _, mu, rs, q = pk.ln_forward(x, gamma, beta, EPS, checkpoint=True)
    src, value = (q, pk.q8_decode(q, torch.float32)) if kept == "q8" else (x, x)
    rdx, rdg, rdb = ref_backward(dy, value, mu, rs, gamma, add)
    h = (value.double() - mu.double()[:, None]) * rs.double()[:, None]
    terms = ((dy.double() * h).abs().sum(0), dy.double().abs().sum(0))
    into = dy.clone()
    dx, dg, db = pk.ln_backward(into, src, mu, rs, gamma, add=add, dx=into)
    near(dx, rdx, TOL[dtype])
    for got, want, t in ((dg, rdg, terms[0]), (db, rdb, terms[1])):
        assert ((got.double() - want).abs() <= 2.0 ** -24 * (rows + 8) * t).all()
