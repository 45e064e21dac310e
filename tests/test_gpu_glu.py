"""The gated linear layer and its gradient against 64-bit references, element by element within the error that fp32
sums of that length may have."""
import math

import pytest
import torch

from test_gpu_linear import GROUP, U, act_pair, product, randn, store, within

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def check_codes(q, z, ez):
    """Scales from the largest |z| of each group; values within half a step of z."""
    rows, F = z.shape
    n = -(-F // GROUP)
    pz, pe = torch.zeros(2, rows, n * GROUP, dtype=torch.float64, device="cuda").unbind(0)
    pz[:, :F], pe[:, :F] = z, ez
    top, etop = pz.view(rows, n, GROUP).abs().amax(2), pe.view(rows, n, GROUP).amax(2)
    within(q.scales, top / 127, (etop + 2 * U * top) / 127)
    step = q.scales.double().repeat_interleave(GROUP, 1)[:, :F]
    within(q.codes.double() * step, z, step * (0.5 + 127 * 8 * U) + ez)


def check_forward(pk, dtype, rows, n_in, F, act, bias=True, pad=0):
    s = rows + 3 * n_in + 7 * F
    x = randn(rows, n_in, dtype=dtype, seed=s, pad=pad)
    W = randn(2 * F, n_in, dtype=dtype, seed=s + 1, scale=1 / math.sqrt(n_in), pad=pad)
    b = randn(2 * F, dtype=dtype, seed=s + 2) if bias else None
    z, ez = product(x, W.t(), n_in)
    if bias:
        z = z + b.double()
        ez = ez + 2 * U * b.double().abs()
    g, u, eg, eu = z[:, :F], z[:, F:], ez[:, :F], ez[:, F:]
    a, _ = act_pair(g, act)
    h = a * u
    # |act'| <= 1.13; act itself within 4 units of |g|; one more product
    ea = 1.13 * eg + 4 * U * g.abs() + 2 * U * a.abs()
    tol = ea * (u.abs() + eu) + a.abs() * eu + 2 * U * h.abs()
    got, none = pk.glu_forward(x, W, b, act)
    assert none is None
    # bf16 forms gelu's tail within 0.75e-7, and silu's exponential within a few units of 2^-23
    tol = tol + (1e-7 * g.abs() * u.abs() if dtype == BF16 else 0)
    within(got, h, tol * (1 + 2.0 ** -8) + store(dtype, h))
    got2, kept = pk.glu_forward(x, W, b, act, keep="z")
    within(got2, h, tol * (1 + 2.0 ** -8) + store(dtype, h))
    within(kept, z, ez * (1 + 2.0 ** -8) + store(dtype, z))
    got3, pair = pk.glu_forward(x, W, b, act, keep="q8")
    within(got3, h, tol * (1 + 2.0 ** -8) + store(dtype, h))
    check_codes(pair[0], g, eg)
    check_codes(pair[1], u, eu)
    again = pk.glu_forward(x, W, b, act, keep="q8")
    assert torch.equal(again[0], got3) and all(torch.equal(p, q) for c, d in zip(again[1], pair) for p, q in zip(c, d))


# one token, one input, one hidden column; tiles filled and not; tails of every kind
SHAPES = [(1, 1, 1), (1, 64, 300), (1, 4096, 512), (3, 7, 5), (17, 100, 129), (16, 256, 256), (64, 96, 500), (128, 256, 64),
          (33, 1000, 77), (257, 264, 200), (300, 513, 130), (512, 2048, 128), (5, 5000, 31), (700, 72, 1024),
          (8, 700, 1030), (9, 520, 130), (12, 4100, 600), (2, 130, 5000), (15, 33, 1025), (40, 600, 65), (65, 130, 191)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n_in,F", SHAPES)
@pytest.mark.parametrize("act,bias,pad", [("silu", True, 0), ("gelu", False, 8), ("relu", True, 3), ("none", True, 2)])
def test_forward(pk, dtype, rows, n_in, F, act, bias, pad):
    check_forward(pk, dtype, rows, n_in, F, act, bias, pad)


# Every tile, whole and cut, and with a checkpoint: (type, rows, n_in, F)
TILES = [(BF16, 20, 2048, 1000), (BF16, 60, 4098, 300), (BF16, 500, 66, 4100), (BF16, 300, 1243, 90), (BF16, 2338, 2119, 1681),
         (BF16, 4100, 1030, 4099), (BF16, 5392, 1251, 1488), (BF16, 5440, 7208, 221), (F32, 20, 450, 150), (F32, 2225, 722, 1360),
         (F32, 1280, 3138, 33), (F32, 4463, 484, 914), (F32, 8452, 706, 225)]


@pytest.mark.parametrize("dtype,rows,n_in,F", TILES)
def test_forward_of_every_tile(pk, dtype, rows, n_in, F):
    check_forward(pk, dtype, rows, n_in, F, "silu")


def check_backward(pk, dtype, rows, n_out, F, act, kept_as, pad=0):
    s = rows + 3 * n_out + 7 * F
    dy = randn(rows, n_out, dtype=dtype, seed=s, pad=pad)
    W = randn(n_out, F, dtype=dtype, seed=s + 1, scale=1 / math.sqrt(n_out), pad=pad)
    z = randn(rows, 2 * F, dtype=dtype, seed=s + 2, pad=pad)
    v = z.double()
    kept = z
    if kept_as == "q8":
        kept = pk.q8_encode(z[:, :F]), pk.q8_encode(z[:, F:])
        v = torch.cat([pk.q8_decode(q, F32) for q in kept], 1).double()
    g, u = v[:, :F], v[:, F:]
    a, slope = act_pair(g, act)
    ea = 4 * U * g.abs() + 2 * U * a.abs() + (1e-7 * g.abs() if dtype == BF16 else 0)
    es = 16 * U * (1 + g.abs()) + (2e-7 if dtype == BF16 else 0)
    dh, eh = product(dy, W, n_out)

    def against(dz, h, dh, eh):
        want = torch.cat((dh * u * slope, dh * a), 1)
        tol = torch.cat((u.abs() * (eh * slope.abs() + (dh.abs() + eh) * es), eh * a.abs() + (dh.abs() + eh) * ea), 1)
        within(dz, want, (tol + 4 * U * want.abs()) * (1 + 2.0 ** -8) + store(dtype, want))
        if h is not None:
            within(h, a * u, (ea * u.abs() + 2 * U * (a * u).abs()) * (1 + 2.0 ** -8) + store(dtype, a * u))
    dz, h, db = pk.glu_backward_input(dy, W, kept, act, hidden=True, bias=True)
    against(dz, h, dh, eh)
    dz2, none, nodb = pk.glu_backward_input(dy, W, kept, act)
    assert none is nodb is None and torch.equal(dz2, dz)
    # sums of what dz is before its rounding, in some order
    want = torch.cat((dh * u * slope, dh * a), 1)
    size = torch.cat((u.abs() * (eh * slope.abs() + (dh.abs() + eh) * es), eh * a.abs() + (dh.abs() + eh) * ea), 1)
    within(db, want.sum(0), (size + U * (rows + 8) * want.abs()).sum(0))
    base = randn(2 * F, dtype=F32, seed=s + 3)
    more = base.clone()
    pk.glu_backward_input(dy, W, kept, act, bias=True, dbias=more, accumulate=True)
    assert torch.equal(more, base + db)
    # of a given dh
    given = dh.to(dtype)
    dz3, h3 = pk.glu_backward_act(given, kept, act, hidden=True)
    against(dz3, h3, given.double(), torch.zeros_like(dh))
    assert torch.equal(h3, h)
    if kept_as == "whole":         # dz in place of z, h in place of dh
        into = z.clone() if not pad else torch.nn.functional.pad(z, (0, pad))[:, :2 * F]
        pk.glu_backward_input(dy, W, into, act, dz=into)
        assert torch.equal(into, dz)
        into, at = z.contiguous(), given.clone()
        pk.glu_backward_act(at, into, act, dz=into, h=at)
        assert torch.equal(into, dz3) and torch.equal(at, h3)


@pytest.mark.parametrize("kept_as", ["whole", "q8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,n_out,F", SHAPES)
def test_backward(pk, dtype, rows, n_out, F, kept_as):
    act = ("silu", "gelu", "relu", "none")[(rows + F) % 4]
    check_backward(pk, dtype, rows, n_out, F, act, kept_as, pad=(0, 8, 3)[rows % 3])


@pytest.mark.parametrize("kept_as", ["whole", "q8"])
@pytest.mark.parametrize("dtype,rows,n_out,F", [(BF16, 9, 6082, 194), (BF16, 34, 1997, 2171), (BF16, 516, 34, 6530),
                                                (BF16, 300, 1474, 50), (BF16, 300, 66, 50), (BF16, 70, 5073, 1067),
                                                (BF16, 1297, 2113, 5930), (BF16, 4610, 4610, 2050), (BF16, 9369, 1171, 1727),
                                                (F32, 9, 436, 300), (F32, 8196, 33, 194), (F32, 1302, 705, 3289),
                                                (F32, 97, 560, 193), (F32, 130, 440, 50), (F32, 4463, 484, 1827)])
def test_backward_of_every_tile(pk, dtype, rows, n_out, F, kept_as):
    check_backward(pk, dtype, rows, n_out, F, "silu", kept_as)


def test_a_non_finite_row_stays_alone(pk):
    for rows in (5, 200):
        x = randn(rows, 300, dtype=BF16, seed=1)
        W = randn(2 * 140, 300, dtype=BF16, seed=2, scale=0.05)
        h, pair = pk.glu_forward(x, W, None, keep="q8")
        bad = x.clone()
        bad[3, 7] = float("nan")
        hb, pb = pk.glu_forward(bad, W, None, keep="q8")
        ok = [i for i in range(rows) if i != 3]
        assert torch.equal(hb[ok], h[ok]) and torch.isnan(hb[3]).all()
        for a, b in zip(pair, pb):
            assert torch.equal(a.codes[ok], b.codes[ok]) and torch.equal(a.scales[ok], b.scales[ok]) and torch.isnan(b.scales[3]).all()


def test_no_rows_and_columns_behind_the_last(pk):
    W = randn(2 * 96, 64, dtype=BF16, seed=2, scale=0.1)
    e = torch.empty(0, 64, dtype=BF16, device="cuda")
    h, z = pk.glu_forward(e, W, None, keep="z")
    assert h.shape == (0, 96) and z.shape == (0, 192)
    dz, h, db = pk.glu_backward_input(e, randn(64, 96, dtype=BF16, seed=3), z, hidden=True, bias=True)
    assert dz.shape == (0, 192) and h.shape == (0, 96) and (db == 0).all()
    for rows in (4, 150):
        x = randn(rows, 64, dtype=BF16, seed=4)
        wide = torch.full((rows + 1, 101), 9.0, dtype=BF16, device="cuda")
        want, _ = pk.glu_forward(x, W, None)
        pk.glu_forward(x, W, None, h=wide[:rows, :96])
        assert torch.equal(wide[:rows, :96], want) and (wide[:, 96:] == 9).all() and (wide[rows] == 9).all()


@pytest.mark.parametrize("rows", [3, 24, 600])
def test_streams_and_graphs(pk, rows):
    """On another stream, and replayed; two graphs with workspaces of their own."""
    n_in, F = 1024, 768
    x, W, b = randn(rows, n_in, dtype=BF16, seed=1), randn(2 * F, n_in, dtype=BF16, seed=2, scale=0.03), randn(2 * F, dtype=BF16, seed=3)
    dy, W2 = randn(rows, n_in, dtype=BF16, seed=4), randn(n_in, F, dtype=BF16, seed=5, scale=0.03)

    def both(s=None):
        h, kept = pk.glu_forward(x, W, b, keep="q8", stream=s)
        return [h, *kept[0], *kept[1], *pk.glu_backward_input(dy, W2, kept, hidden=True, bias=True, stream=s)]
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graphs, held = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for g in graphs:
        with torch.cuda.graph(g):
            held.append(both())
    for i in range(3):
        x.copy_(torch.randn(rows, n_in, device="cuda"))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = both()
        assert all(torch.equal(p, q) for h in held for p, q in zip(h, want))


def test_workspace_and_refusals_on_the_device(pk):
    x, W = randn(40, 2048, dtype=BF16, seed=1), randn(256, 2048, dtype=BF16, seed=2)
    need = pk.glu_workspace_size(pk.GLU_FORWARD, 40, 2048, 128, BF16)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert torch.equal(pk.glu_forward(x, W, ws=ws)[0], pk.glu_forward(x, W)[0])
    with pytest.raises(pk.AcscError, match="needed"):
        pk.glu_forward(x, W, ws=ws[:need // 2])
    with pytest.raises(pk.AcscError, match="even"):
        pk.glu_forward(x, W[:255])
    with pytest.raises(pk.AcscError, match="keep"):
        pk.glu_forward(x, W, keep="both")
    h, z = pk.glu_forward(x, W, keep="z")
    with pytest.raises(pk.AcscError, match="pair"):
        pk.glu_backward_act(h, pk.q8_encode(z))
    with pytest.raises(pk.AcscError, match="z must be"):
        pk.glu_backward_act(h, z[:, :128])
    with pytest.raises(pk.AcscError, match="overlap"):
        pk.glu_forward(x, W, h=x[:, :128])


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows", [2, 40])
def test_gates_at_the_ends_of_the_range(pk, act, dtype, rows):
    """Gates that all but close, times large up values: h and its gradient keep their relative accuracy as far as the
    activation of a linear layer does."""
    g = torch.tensor([-95.0, -89.0, -88.0, -80.0, -40.0, -13.0, -5.0, 0.0, 5.0, 40.0, 89.0, 1e4]).to(dtype).cuda()
    F = g.numel()
    # z = x W' + b of x = 1 and W = 0
    x = torch.ones(rows, 8, dtype=dtype, device="cuda")
    W = torch.zeros(2 * F, 8, dtype=dtype, device="cuda")
    big = torch.full((F,), 1e30, dtype=dtype, device="cuda")
    big[-1] = 1.0
    h, z = pk.glu_forward(x, W, torch.cat((g, big)), act, keep="z")
    a = pk.lin_forward(x, W[:F], g, act)[0].double()
    want = a * big.double()
    # one rounding of a and one of h more than the exact product has
    eps = 2.0 ** -7 if dtype == BF16 else 2.0 ** -22
    assert ((h.double() - want).abs() <= eps * want.abs() + 1e-8).all()
    dz, _ = pk.glu_backward_act(torch.ones_like(h), z, act)
    assert ((dz[:, F:].double() - a).abs() <= eps * a.abs() + 1e-38).all()
    slope = pk.lin_backward_act(torch.ones_like(h), z[:, :F].contiguous(), act).double()
    assert ((dz[:, :F].double() - slope * big.double()).abs() <= eps * (slope * big.double()).abs() + 1e-8).all()
