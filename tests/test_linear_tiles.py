"""Every tile of the linear layers' products, whole, cut along the sum, and whole with a cut rest: that the shapes
below reach them (host only), and their results against 64-bit references."""
import pytest
import torch

from test_gpu_linear import GROUP, U, act_pair, product, store, within

BF16, F32 = torch.bfloat16, torch.float32
FORWARD, INPUT, WEIGHT = 0, 1, 2

# (type, product, tile, whole tiles, cut tiles, (rows, n_in, n_out)): ragged ones, at least two tiles each way where
# there are many; rows of whole and of part chunks
CASES = [
    (BF16, FORWARD, (32, 128), False, True, (9, 4034, 130)),
    (BF16, FORWARD, (64, 128), False, True, (35, 1789, 2479)),
    (BF16, FORWARD, (64, 128), True, False, (399, 34, 8478)),
    (BF16, FORWARD, (128, 64), False, True, (300, 1474, 50)),
    (BF16, FORWARD, (128, 64), True, False, (300, 66, 50)),
    (BF16, FORWARD, (128, 128), False, True, (70, 1243, 167)),
    (BF16, FORWARD, (128, 128), True, False, (270, 130, 300)),
    (BF16, FORWARD, (128, 128), True, True, (2338, 2119, 3362)),
    (BF16, FORWARD, (256, 256), False, True, (5440, 7208, 442)),
    (BF16, FORWARD, (256, 256), True, False, (4100, 1030, 8198)),
    (BF16, FORWARD, (256, 256), True, True, (5392, 1251, 2975)),
    (BF16, INPUT, (32, 128), False, True, (9, 194, 6082)),
    (BF16, INPUT, (64, 128), False, True, (34, 2171, 1997)),
    (BF16, INPUT, (64, 128), True, False, (516, 6530, 34)),
    (BF16, INPUT, (128, 64), False, True, (300, 50, 1474)),
    (BF16, INPUT, (128, 64), True, False, (300, 50, 66)),
    (BF16, INPUT, (128, 128), False, True, (70, 1067, 5073)),
    (BF16, INPUT, (128, 128), True, False, (129, 8755, 34)),
    (BF16, INPUT, (128, 128), True, True, (1297, 5930, 2113)),
    (BF16, INPUT, (256, 256), False, True, (4100, 1030, 8198)),
    (BF16, INPUT, (256, 256), True, False, (4610, 2050, 4610)),
    (BF16, INPUT, (256, 256), True, True, (9369, 1727, 1171)),
    (BF16, WEIGHT, (64, 128), False, True, (1792, 1474, 34)),
    (BF16, WEIGHT, (64, 128), True, False, (40, 8194, 386)),
    (BF16, WEIGHT, (128, 64), False, True, (1479, 34, 300)),
    (BF16, WEIGHT, (128, 64), True, False, (99, 34, 300)),
    (BF16, WEIGHT, (128, 128), False, True, (4612, 66, 1026)),
    (BF16, WEIGHT, (128, 128), True, False, (40, 8194, 130)),
    (BF16, WEIGHT, (128, 128), True, True, (1796, 2387, 3343)),
    (BF16, WEIGHT, (256, 256), False, True, (7551, 389, 5836)),
    (BF16, WEIGHT, (256, 256), True, False, (4610, 2050, 4610)),
    (BF16, WEIGHT, (256, 256), True, True, (1280, 2434, 6594)),
    (F32, FORWARD, (32, 128), False, True, (20, 450, 300)),
    (F32, FORWARD, (32, 128), True, False, (8196, 33, 130)),
    (F32, FORWARD, (32, 128), True, True, (8452, 706, 450)),
    (F32, FORWARD, (64, 128), False, True, (111, 422, 140)),
    (F32, FORWARD, (64, 128), True, False, (70, 67, 130)),
    (F32, FORWARD, (64, 128), True, True, (2225, 722, 2720)),
    (F32, FORWARD, (128, 64), False, True, (130, 440, 50)),
    (F32, FORWARD, (128, 128), False, True, (1280, 3138, 66)),
    (F32, FORWARD, (128, 128), True, False, (8196, 34, 258)),
    (F32, FORWARD, (128, 128), True, True, (4463, 484, 1827)),
    (F32, INPUT, (32, 128), False, True, (9, 300, 436)),
    (F32, INPUT, (32, 128), True, False, (8196, 194, 33)),
    (F32, INPUT, (32, 128), True, True, (1302, 3289, 705)),
    (F32, INPUT, (64, 128), False, True, (97, 193, 560)),
    (F32, INPUT, (64, 128), True, False, (70, 130, 67)),
    (F32, INPUT, (64, 128), True, True, (3076, 1986, 706)),
    (F32, INPUT, (128, 64), False, True, (130, 50, 440)),
    (F32, INPUT, (128, 64), True, False, (8196, 130, 34)),
    (F32, INPUT, (128, 64), True, True, (3332, 1154, 642)),
    (F32, INPUT, (128, 128), False, True, (1280, 66, 3074)),
    (F32, INPUT, (128, 128), True, False, (8196, 258, 34)),
    (F32, INPUT, (128, 128), True, True, (2851, 2863, 485)),
    (F32, WEIGHT, (64, 128), False, True, (441, 141, 131)),
    (F32, WEIGHT, (64, 128), True, False, (67, 130, 70)),
    (F32, WEIGHT, (64, 128), True, True, (718, 8208, 705)),
    (F32, WEIGHT, (128, 64), False, True, (512, 50, 200)),
    (F32, WEIGHT, (128, 64), True, False, (33, 130, 8194)),
    (F32, WEIGHT, (128, 64), True, True, (629, 3696, 1126)),
    (F32, WEIGHT, (128, 128), False, True, (3332, 1090, 66)),
    (F32, WEIGHT, (128, 128), True, False, (33, 8194, 194)),
    (F32, WEIGHT, (128, 128), True, True, (512, 962, 8258)),
]
IDS = ["-".join(map(str, (str(c[0])[6:], "fwd dx dw".split()[c[1]], "%dx%d" % c[2], "whole" * c[3] + "cut" * c[4])))
       for c in CASES]


@pytest.fixture(scope="module")
def pk():
    import paper_2609_14339_amd as pk
    return pk


@pytest.mark.parametrize("dtype,op,tile,whole,cut,shape", CASES, ids=IDS)
def test_the_plan(pk, dtype, op, tile, whole, cut, shape):
    p = pk.lin_product_plan(op, *shape, dtype)
    assert (p.tile_rows, p.tile_cols) == tile and (p.whole > 0) == whole and (p.cut > 0) == cut and (p.pieces > 1) == cut
    rows, n_in, n_out = shape
    M, N = {FORWARD: (rows, n_out), INPUT: (rows, n_in), WEIGHT: (n_out, n_in)}[op]
    assert p.whole + p.cut == -(-M // tile[0]) * -(-N // tile[1])


def test_plans_of_few_rows_and_refusals(pk):
    assert pk.lin_product_plan(FORWARD, 1, 4096, 4096, BF16)[:4] == (0, 0, 0, 0)
    assert pk.lin_product_plan(WEIGHT, 8, 4096, 4096, F32) == (0, 0, 0, 0, 1)
    assert pk.lin_product_plan(INPUT, 0, 64, 64, F32) == (0, 0, 0, 0, 0)
    for bad in ((3, 1, 1, 1), (0, -1, 1, 1), (0, 1, 0, 1), (0, 1 << 30, 1 << 22, 1 << 22)):
        with pytest.raises(pk.AcscError):
            pk.lin_product_plan(*bad, BF16)
    assert pk.lib.lin_product_plan(0, 1, 1, 1, 0, None) == -1


def randn(g, *shape, dtype, scale=1.0):
    return torch.randn(*shape, generator=g, device="cuda").mul_(scale).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,op,tile,whole,cut,shape", CASES, ids=IDS)
def test_the_product(pk, dtype, op, tile, whole, cut, shape):
    """With every part of the epilogue: bias, activation, residual and checkpoint; the gate from a checkpoint and from a
    tensor; a gradient that is added to, from a checkpoint and from a tensor.  The bounds are those of the other tests
    of these products."""
    rows, n_in, n_out = shape
    g = torch.Generator(device="cuda").manual_seed(rows + n_in)
    W = randn(g, n_out, n_in, dtype=dtype, scale=n_in ** -0.5)
    if op == FORWARD:
        x, b, r = randn(g, rows, n_in, dtype=dtype), randn(g, n_out, dtype=dtype), randn(g, rows, n_out, dtype=dtype)
        z, ez = product(x, W.t(), n_in)
        z, ez = z + b.double(), ez + 2 * U * b.double().abs()
        a, _ = act_pair(z, "gelu")
        y = a + r.double()
        got, q = pk.lin_forward(x, W, b, "gelu", r, keep="q8")
        within(got, y, (1.13 * ez + 4 * U * z.abs() + 2 * U * (a.abs() + y.abs())) * (1 + 2.0 ** -8) + store(dtype, y))
        step = q.scales.double().repeat_interleave(GROUP, 1)[:, :n_out]
        within(q.codes.double() * step, z, step * (0.5 + 127 * 8 * U) + ez)
        again, kept = pk.lin_forward(x, W, b, "gelu", r, keep="z")
        assert torch.equal(again, got)
        within(kept, z, ez * (1 + 2.0 ** -8) + store(dtype, z))
        return
    dz, z = randn(g, rows, n_out, dtype=dtype), randn(g, rows, n_in, dtype=dtype)
    q = pk.q8_encode(z)
    if op == INPUT:
        p, ep = product(dz, W, n_out)
        for src, v in ((z, z.double()), (q, pk.q8_decode(q, F32).double())):
            want = p * act_pair(v, "silu")[1]
            tol = ep * 1.13 + 8 * U * p.abs() + 2 * U * want.abs()
            within(pk.lin_backward_input(dz, W, "silu", src), want, tol * (1 + 2.0 ** -8) + store(dtype, want))
        within(pk.lin_backward_input(dz, W), p, ep * (1 + 2.0 ** -8) + store(dtype, p))
        return
    db64, db_tol = dz.double().sum(0), 2 * U * (rows + 8) * dz.double().abs().sum(0)
    for src, v, act in ((z, z.double(), "none"), (q, pk.q8_decode(q, F32).double(), "gelu")):
        a, _ = act_pair(v, act)
        ea = torch.zeros_like(a) if act == "none" else 4 * U * v.abs() + 2 * U * a.abs() + store(dtype, a) * (1 + 2.0 ** -8)
        p, ep = product(dz.t(), a, rows)
        ep = ep * (1 + 2.0 ** -7) + dz.double().abs().t() @ ea
        for dw_dtype in (BF16, F32):
            dW, db = pk.lin_backward_weight(dz, src, act, dw_dtype=dw_dtype)
            within(dW, p, ep * (1 + 2.0 ** -8) + store(dw_dtype, p))
            within(db, db64, db_tol)
        sw, sb = randn(g, n_out, n_in, dtype=F32), randn(g, n_out, dtype=F32)
        aw, ab = sw.clone(), sb.clone()
        pk.lin_backward_weight(dz, src, act, dW=aw, db=ab, accumulate=True)
        assert torch.equal(aw, sw + dW) and torch.equal(ab, sb + db)
