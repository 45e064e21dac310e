"""Fused linear layers and their gradients against 64-bit references, element
by element within the error that fp32 sums of that length may have."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
GROUP = 128
U = 2.0 ** -24
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def act_pair(z, act):
    """(act, act') in 64 bits."""
    if act == "relu":
        return z.clamp_min(0), (z > 0).double()
    if act == "gelu":
        phi = 0.5 * torch.erfc(-z / math.sqrt(2))
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * (1 - s))
    return z, torch.ones_like(z)


def store(dtype, ref):
    """What storing a value of about ref may add: half a unit in the last of bf16's 8 significant bits, or of fp32's 24."""
    return ref.abs() * (2.0 ** -8 if dtype == BF16 else U)


def within(got, want, tol):
    got, want, tol = got.double().cpu(), want.cpu(), tol.cpu()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - tol - 1e-36
    assert (over <= 0).all(), f"{int((over > 0).sum())} of {over.numel()} out of bounds, by up to {float(over.max()):.3e}"


def randn(*shape, dtype, seed, scale=1.0, pad=0):
    g = torch.Generator().manual_seed(seed)
    t = torch.randn(*shape[:-1], shape[-1] + pad, generator=g).mul_(scale).to(dtype).cuda()
    return t[..., :shape[-1]]


def product(a, b, n):
    """a b in 64 bits, and the bound of an fp32 sum of n products in any order: each product and each addition off by
    at most a unit of 2^-23 (the matrix cores may cut where others round)."""
    a, b = a.double(), b.double()
    return a @ b, 2 * U * (n + 8) * (a.abs() @ b.abs())


# (rows, n_in, n_out): one token, one input, one output, tiles filled and not, k tails of every kind, many pieces
SHAPES = [(1, 1, 1), (1, 64, 300), (1, 4096, 512), (3, 7, 5), (17, 100, 129), (16, 256, 256), (64, 96, 1000),
          (128, 256, 128), (33, 1000, 77), (257, 264, 392), (300, 513, 260), (512, 2048, 256), (5, 5000, 31),
          (700, 72, 1024),
          # few tokens: the products that do not tile them, at their limits and past
          (8, 700, 1030), (9, 520, 130), (12, 4100, 600), (2, 130, 5000), (15, 33, 1025)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
@pytest.mark.parametrize("act,full,pad", [("none", False, 0), ("gelu", True, 0), ("silu", True, 8), ("relu", True, 3)])
def test_forward(pk, dtype, rows, n_in, n_out, act, full, pad):
    s = rows + 3 * n_in + 7 * n_out
    x = randn(rows, n_in, dtype=dtype, seed=s, pad=pad)
    W = randn(n_out, n_in, dtype=dtype, seed=s + 1, scale=1 / math.sqrt(n_in), pad=pad)
    b = randn(n_out, dtype=dtype, seed=s + 2) if full else None
    r = randn(rows, n_out, dtype=dtype, seed=s + 3, pad=pad) if full else None
    z, ez = product(x, W.t(), n_in)
    if full:
        z = z + b.double()
        ez = ez + 2 * U * b.double().abs()
    a, _ = act_pair(z, act)
    y = a + (r.double() if full else 0)
    # |act'| <= 1.13; act itself within 4 units of |z|; one more addition
    tol = 1.13 * ez + 4 * U * z.abs() + 2 * U * (a.abs() + y.abs())
    got, none = pk.lin_forward(x, W, b, act, r)
    assert none is None
    within(got, y, tol * (1 + 2.0 ** -8) + store(dtype, y))
    got2, zz = pk.lin_forward(x, W, b, act, r, keep="z")
    assert torch.equal(got2, got)
    within(zz, z, ez * (1 + 2.0 ** -8) + store(dtype, z))
    got3, q = pk.lin_forward(x, W, b, act, r, keep="q8")
    assert torch.equal(got3, got)
    # the checkpoint: scales from the largest |z| of each group; values within half a step of z
    n = -(-n_out // GROUP)
    pz, pe = torch.zeros(2, rows, n * GROUP, dtype=torch.float64, device="cuda").unbind(0)
    pz[:, :n_out], pe[:, :n_out] = z, ez
    top = pz.view(rows, n, GROUP).abs().amax(2)
    etop = pe.view(rows, n, GROUP).amax(2)
    within(q.scales, top / 127, (etop + 2 * U * top) / 127)
    step = q.scales.double().repeat_interleave(GROUP, 1)[:, :n_out]
    within(q.codes.double() * step, z, step * (0.5 + 127 * 8 * U) + ez)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [7, 10, 16, 17, 32, 33, 50, 64, 65, 97, 130])
@pytest.mark.parametrize("n_in,n_out,pad", [(4104, 1160, 0), (1160, 4104, 8), (2053, 771, 3)])
def test_few_rows(pk, dtype, rows, n_in, n_out, pad):
    """The forward product and the input gradient of few tokens on wide layers: narrow tiles, whole and cut, one and
    several of them, their last rows and columns part full; operands of odd strides copied or read where they are."""
    s = rows + n_in
    x = randn(rows, n_in, dtype=dtype, seed=s, pad=pad)
    W = randn(n_out, n_in, dtype=dtype, seed=s + 1, scale=1 / math.sqrt(n_in), pad=pad)
    b, r = randn(n_out, dtype=dtype, seed=s + 2), randn(rows, n_out, dtype=dtype, seed=s + 3, pad=pad)
    z, ez = product(x, W.t(), n_in)
    z, ez = z + b.double(), ez + 2 * U * b.double().abs()
    a, _ = act_pair(z, "silu")
    y = a + r.double()
    got, q = pk.lin_forward(x, W, b, "silu", r, keep="q8")
    within(got, y, (1.13 * ez + 4 * U * z.abs() + 2 * U * (a.abs() + y.abs())) * (1 + 2.0 ** -8) + store(dtype, y))
    step = q.scales.double().repeat_interleave(GROUP, 1)[:, :n_out]
    within(q.codes.double() * step, z, step * (0.5 + 127 * 8 * U) + ez)
    for again in (pk.lin_forward(x, W, b, "silu", r), pk.lin_forward(x, W, b, "silu", r, keep="z")):
        assert torch.equal(again[0], got)
    within(again[1], z, ez * (1 + 2.0 ** -8) + store(dtype, z))
    dz, kept = randn(rows, n_out, dtype=dtype, seed=s + 4, pad=pad), randn(rows, n_in, dtype=dtype, seed=s + 5, pad=pad)
    p, ep = product(dz, W, n_out)
    within(pk.lin_backward_input(dz, W), p, ep * (1 + 2.0 ** -8) + store(dtype, p))
    code = pk.q8_encode(kept)
    for src, v in ((kept, kept.double()), (code, pk.q8_decode(code, F32).double())):
        want = p * act_pair(v, "silu")[1]
        tol = ep * 1.13 + 8 * U * p.abs() + 2 * U * want.abs()
        within(pk.lin_backward_input(dz, W, "silu", src), want, tol * (1 + 2.0 ** -8) + store(dtype, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [33, 65, 130, 1100])
@pytest.mark.parametrize("n_in,n_out,pad", [(1, 64, 0), (2, 3, 0), (3, 2, 0), (5, 33, 1), (64, 1000, 0), (2051, 64, 0), (4100, 50, 2),
                                            (50, 4100, 2), (66, 130, 4)])
def test_narrow_layers(pk, dtype, rows, n_in, n_out, pad):
    """Few inputs or outputs: tiles of 64 columns, whole and cut; rows that are shorter than a 16-byte chunk or end inside
    one, and sums that do."""
    s = rows + n_in
    x = randn(rows, n_in, dtype=dtype, seed=s, pad=pad)
    W = randn(n_out, n_in, dtype=dtype, seed=s + 1, scale=1 / math.sqrt(n_in), pad=pad)
    dz = randn(rows, n_out, dtype=dtype, seed=s + 2, pad=pad)
    z, ez = product(x, W.t(), n_in)
    got, q = pk.lin_forward(x, W, keep="q8")
    within(got, z, ez * (1 + 2.0 ** -8) + store(dtype, z))
    n = -(-n_out // GROUP)
    pz, pe = torch.zeros(2, rows, n * GROUP, dtype=torch.float64, device="cuda").unbind(0)
    pz[:, :n_out], pe[:, :n_out] = z, ez
    top = pz.view(rows, n, GROUP).abs().amax(2)
    within(q.scales, top / 127, (pe.view(rows, n, GROUP).amax(2) + 2 * U * top) / 127)
    step = q.scales.double().repeat_interleave(GROUP, 1)[:, :n_out]
    within(q.codes.double() * step, z, step * (0.5 + 127 * 8 * U) + ez)
    p, ep = product(dz, W, n_out)
    within(pk.lin_backward_input(dz, W), p, ep * (1 + 2.0 ** -8) + store(dtype, p))
    p, ep = product(dz.t(), x, rows)
    for dw_dtype in (BF16, F32):
        dW, db = pk.lin_backward_weight(dz, x, dw_dtype=dw_dtype)
        within(dW, p, ep * (1 + 2.0 ** -8) + store(dw_dtype, p))
        within(db, dz.double().sum(0), 2 * U * (rows + 8) * dz.double().abs().sum(0))
    # operands that end with the memory they were given: the last rows of a larger tensor
    base = randn(rows + 9, n_in, dtype=dtype, seed=s + 3)
    assert torch.equal(pk.lin_forward(base[9:], W)[0], pk.lin_forward(base[9:].clone(), W)[0])


@pytest.mark.parametrize("kept", ["z", "q8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n_in,n_out", SHAPES)
@pytest.mark.parametrize("act,pad", [("none", 0), ("gelu", 8), ("silu", 0), ("relu", 5)])
def test_backward(pk, dtype, rows, n_in, n_out, act, pad, kept):
    s = rows + 3 * n_in + 7 * n_out + 11
    dz = randn(rows, n_out, dtype=dtype, seed=s, pad=pad)
    W = randn(n_out, n_in, dtype=dtype, seed=s + 1, scale=1 / math.sqrt(n_in), pad=pad)
    z = randn(rows, n_in, dtype=dtype, seed=s + 2, pad=pad)
    src, zv = z, z.double()
    if kept == "q8":
        src = pk.q8_encode(z)
        zv = pk.q8_decode(src, F32).double()
    a, slope = act_pair(zv, act)
    # input gradient; act' within 8 units (|z phi(z)| and s |z| (1 - s) stay under 0.25)
    p, ep = product(dz, W, n_out)
    want = p * slope
    tol = ep * 1.13 + 8 * U * p.abs() + 2 * U * want.abs()
    got = pk.lin_backward_input(dz, W, act, src if act != "none" else None)
    within(got, want, tol * (1 + 2.0 ** -8) + store(dtype, want))
    # weight gradient; the activation recomputed and rounded to the tensors' type
    ea = (4 * U * zv.abs() + 2 * U * a.abs()) + store(dtype, a) * (1 + 2.0 ** -8)
    if kept == "z" and act in ("none", "relu"):
        ea = torch.zeros_like(ea)          # nothing is rounded
    pw, ew = product(dz.t(), a, rows)
    ew = ew * (1 + 2.0 ** -7) + dz.double().abs().t() @ ea
    db_tol = 2 * U * (rows + 8) * dz.double().abs().sum(0)
    for dw_dtype in (BF16, F32):
        dW, db = pk.lin_backward_weight(dz, src, act, dw_dtype=dw_dtype)
        assert dW.dtype == dw_dtype
        within(dW, pw, ew * (1 + 2.0 ** -8) + store(dw_dtype, pw))
        within(db, dz.double().sum(0), db_tol)
    dW2, none = pk.lin_backward_weight(dz, src, act, dw_dtype=F32, bias=False)
    assert none is None and torch.equal(dW2, dW)
    # gradient accumulation adds to what is there
    sw, sb = torch.randn_like(dW), torch.randn_like(db)
    aw, ab = sw.clone(), sb.clone()
    pk.lin_backward_weight(dz, src, act, dW=aw, db=ab, accumulate=True)
    assert torch.equal(aw, sw + dW) and torch.equal(ab, sb + db)
    # the activation's gradient alone
    g = randn(rows, n_in, dtype=dtype, seed=s + 4, pad=pad)
    want = g.double() * slope
    got = pk.lin_backward_act(g, src, act)
    within(got, want, 8 * U * g.double().abs() + 2 * U * want.abs() + store(dtype, want) * (1 + 2.0 ** -8))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_products_that_fill_many_tiles(pk, dtype):
    """Whole and ragged grids of the largest tiles, against 64-bit products on the GPU."""
    for rows, n_in, n_out in ((2048, 1024, 1536), (1111, 808, 2000), (4097, 320, 520)):
        x = randn(rows, n_in, dtype=dtype, seed=1)
        W = randn(n_out, n_in, dtype=dtype, seed=2, scale=1 / math.sqrt(n_in))
        z, ez = product(x, W.t(), n_in)
        within(pk.lin_forward(x, W)[0], z, ez * (1 + 2.0 ** -8) + store(dtype, z))
        dz = randn(rows, n_out, dtype=dtype, seed=3)
        p, ep = product(dz, W, n_out)
        within(pk.lin_backward_input(dz, W), p, ep * (1 + 2.0 ** -8) + store(dtype, p))
        p, ep = product(dz.t(), x, rows)
        dW, db = pk.lin_backward_weight(dz, x, dw_dtype=F32)
        within(dW, p, ep + store(F32, p))
        within(db, dz.double().sum(0), 2 * U * (rows + 8) * dz.double().abs().sum(0))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n_in,n_out", [(40, 200, 300), (600, 520, 264)])
def test_non_finite_values_stay_in_their_rows(pk, dtype, rows, n_in, n_out):
    x = randn(rows, n_in, dtype=dtype, seed=1)
    W = randn(n_out, n_in, dtype=dtype, seed=2)
    y0 = pk.lin_forward(x, W)[0]
    x[7, n_in - 1] = float("inf")
    x[rows - 1, 0] = float("nan")
    y, q = pk.lin_forward(x, W, keep="q8")
    keep = [r for r in range(rows) if r not in (7, rows - 1)]
    assert torch.equal(y[keep], y0[keep])
    assert torch.isinf(y[7]).all() and torch.isnan(y[rows - 1]).all()
    v = pk.q8_decode(q, F32)
    assert torch.isnan(v[7]).all() and torch.isnan(v[rows - 1]).all() and torch.isfinite(v[keep]).all()
    # a column of W, then a token's gradient
    dz = randn(rows, n_out, dtype=dtype, seed=3)
    d0 = pk.lin_backward_input(dz, W)
    V = W.clone()
    V[n_out - 1, 5] = float("nan")
    d = pk.lin_backward_input(dz, V)
    cols = [c for c in range(n_in) if c != 5]
    assert torch.equal(d[:, cols], d0[:, cols]) and torch.isnan(d[:, 5]).all()
    w0, _ = pk.lin_backward_weight(dz, randn(rows, n_in, dtype=dtype, seed=1))
    dz[rows - 1, 3] = float("inf")
    w, db = pk.lin_backward_weight(dz, randn(rows, n_in, dtype=dtype, seed=1))
    outs = [c for c in range(n_out) if c != 3]
    assert torch.equal(w[outs], w0[outs]) and not torch.isfinite(w[3]).any() and torch.isinf(db[3])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [2, 200])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_activations_at_the_ends_of_the_range(pk, dtype, rows, act):
    """The formulas' values at infinities and NaN, and where exponentials leave the range."""
    nan, inf = float("nan"), float("inf")
    z = torch.tensor([inf, -inf, nan, 0.0, 1e30, -1e30, 65.0, -65.0, 64.0, -64.0, 200.0, -200.0])
    want = dict(none=[inf, -inf, nan, 0, 1e30, -1e30, 65, -65, 64, -64, 200, -200],
                relu=[inf, 0, nan, 0, 1e30, 0, 65, 0, 64, 0, 200, 0],
                gelu=[inf, nan, nan, 0, 1e30, 0, 65, 0, 64, 0, 200, 0],
                silu=[inf, nan, nan, 0, 1e30, 0, 65, 0, 64, 0, 200, 0])[act]
    want = torch.tensor(want).to(dtype).expand(rows, -1)
    x, W = torch.zeros(rows, 40, dtype=dtype, device="cuda"), torch.zeros(12, 40, dtype=dtype, device="cuda")
    got = pk.lin_forward(x, W, z.to(dtype).cuda(), act)[0].cpu()
    # silu(-64) = -64 e^-64 and silu(-65) are numbers of fp32 below 2^-86
    assert torch.allclose(got.float(), want.float(), rtol=0, atol=2.0 ** -86, equal_nan=True)


def test_outputs_in_place_and_margins(pk):
    rows, n_in, n_out = 70, 136, 200
    x = randn(rows, n_in, dtype=BF16, seed=1)
    W = randn(n_out, n_in, dtype=BF16, seed=2)
    r = randn(rows, n_out, dtype=BF16, seed=3)
    want = pk.lin_forward(x, W, residual=r, act="gelu")[0]
    into = r.clone()
    pk.lin_forward(x, W, residual=into, act="gelu", y=into)
    assert torch.equal(into, want)
    wide = torch.full((rows, n_out + 6), 9.0, dtype=BF16, device="cuda")
    pk.lin_forward(x, W, residual=r, act="gelu", y=wide[:, 1:1 + n_out])
    assert torch.equal(wide[:, 1:1 + n_out], want)
    assert (wide[:, 0] == 9).all() and (wide[:, 1 + n_out:] == 9).all()
    dz = randn(rows, n_out, dtype=BF16, seed=4)
    z = randn(rows, n_out, dtype=BF16, seed=5)
    want = pk.lin_backward_act(dz, z, "silu")
    into = dz.clone()
    pk.lin_backward_act(into, z, "silu", dz=into)
    assert torch.equal(into, want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_the_same_call_gives_the_same_bits(pk, dtype):
    x = randn(300, 4000, dtype=dtype, seed=1)
    W = randn(130, 4000, dtype=dtype, seed=2)
    dz = randn(300, 130, dtype=dtype, seed=3)
    a = [pk.lin_forward(x, W)[0], pk.lin_backward_input(dz, W), *pk.lin_backward_weight(dz, x)]
    for _ in range(3):
        b = [pk.lin_forward(x, W)[0], pk.lin_backward_input(dz, W), *pk.lin_backward_weight(dz, x)]
        assert all(torch.equal(s, t) for s, t in zip(a, b))


def test_another_stream_and_a_caller_workspace(pk):
    x = randn(256, 4096, dtype=BF16, seed=1)
    W = randn(512, 4096, dtype=BF16, seed=2)
    want = pk.lin_forward(x, W, act="silu")[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    outs = [pk.lin_forward(x, W, act="silu", stream=side)[0] for _ in range(4)]
    ws = torch.empty(max(256, pk.lin_workspace_size(pk.LIN_FORWARD, 256, 4096, 512, BF16)), dtype=torch.uint8,
                     device="cuda")
    side.synchronize()
    for o in outs:
        assert torch.equal(o, want)
    ws.fill_(255)                                    # what a workspace holds does not matter
    assert torch.equal(pk.lin_forward(x, W, act="silu", ws=ws)[0], want)


def test_replayed_from_a_graph(pk):
    x = randn(64, 2048, dtype=BF16, seed=1)
    W = randn(256, 2048, dtype=BF16, seed=2)
    dz = randn(64, 256, dtype=BF16, seed=3)

    def step():
        y, q = pk.lin_forward(x, W, act="gelu", keep="q8")
        return [y, q.codes, q.scales, pk.lin_backward_input(dz, W), *pk.lin_backward_weight(dz, x)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(3):
        x.copy_(randn(64, 2048, dtype=BF16, seed=10 + i))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_no_rows(pk):
    e, W = torch.empty(0, 24, dtype=BF16, device="cuda"), randn(40, 24, dtype=BF16, seed=1)
    y, q = pk.lin_forward(e, W, keep="q8")
    assert y.shape == (0, 40) and q.codes.shape == (0, 40)
    assert pk.lin_backward_input(y, W).shape == (0, 24)
    dW, db = pk.lin_backward_weight(y, e)
    assert (dW == 0).all() and (db == 0).all() and dW.shape == (40, 24)
    one, two = torch.ones(40, 24, device="cuda"), torch.ones(40, device="cuda")
    pk.lin_backward_weight(y, e, dW=one, db=two, accumulate=True)
    assert (one == 1).all() and (two == 1).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_row_offsets_past_32_bits(pk, dtype):
    ld = (1 << 31) // (2 if dtype == F32 else 1) + 264
    buf = torch.empty(2 * ld + 256, dtype=dtype, device="cuda")
    x = torch.as_strided(buf, (3, 256), (ld, 1))
    src, W = randn(3, 256, dtype=dtype, seed=1), randn(128, 256, dtype=dtype, seed=2)
    x.copy_(src)
    assert torch.equal(pk.lin_forward(x, W)[0], pk.lin_forward(src, W)[0])
    dz = randn(3, 128, dtype=dtype, seed=3)
    assert torch.equal(pk.lin_backward_weight(dz, x)[0], pk.lin_backward_weight(dz, src)[0])
    pk.lin_backward_input(dz, W, dx=x)
    assert torch.equal(x, pk.lin_backward_input(dz, W))
