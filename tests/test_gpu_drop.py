"""Dropout from the step's key: its mask against the oracle's draws, its values, and the calls it allows."""
import numpy as np
import pytest
import torch

from oracle import mask as om

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
M64 = (1 << 64) - 1
FIELDS = dict(seed=0x123456789ABCDEF, layer=7, step=1 << 40, microbatch=3)


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def mix64(z):
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & M64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & M64
    return z ^ (z >> 31)


def drop_key(rows, H, site, B=1, **fields):
    """The chain over the fields (the oracle's), one step on."""
    f = {**FIELDS, **fields}
    k = om.mask_key(f["seed"], f["layer"], f["step"], f["microbatch"], B, rows // B, H)
    return mix64(((k ^ (0x64726F70 << 32 | site)) + 0x9E3779B97F4A7C15) & M64)


def kept(rows, H, p, site, first=0, count=None, B=1, **fields):
    """Where a value is kept, [count, H], by the oracle's draws (numpy here: its loop is checked against it below)."""
    key, T = drop_key(rows, H, site, B=B, **fields), om.bern_threshold(1 - p)
    count = rows if count is None else count
    out = np.zeros((count, H), dtype=bool)
    q = np.arange((H + 1) // 2, dtype=np.uint32)

    def fmix(h):
        h = (h ^ (h >> np.uint32(16))) * np.uint32(0x85EBCA6B)
        h = (h ^ (h >> np.uint32(13))) * np.uint32(0xC2B2AE35)
        return h ^ (h >> np.uint32(16))
    for r in range(count):
        k = om.row_key(key, first + r)
        h = fmix(fmix(np.uint32(k & 0xFFFFFFFF) ^ q) ^ np.uint32(k >> 32))
        out[r] = np.stack((h & np.uint32(0xFFFF), h >> np.uint32(16)), 1).reshape(-1)[:H] < T
    return torch.from_numpy(out), np.float32(65536.0) / np.float32(T)


def make(pk, rows, H, p, site=0, B=1, **fields):
    return pk.Drop(p, pk.make_key(B=B, S=rows // B, H=H, **{**FIELDS, **fields}), site)


def test_the_draws_are_the_oracles():
    rows, H, p = 5, 301, 0.3
    dense = om.bern_mask_dense(drop_key(rows, H, 9), rows, H, 1 - p)
    assert np.array_equal(kept(rows, H, p, 9)[0].numpy(), dense.astype(bool))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,H,pad", [(1, 1, 0), (3, 7, 0), (64, 256, 0), (5, 513, 3), (129, 2051, 5), (2, 70000, 0)])
@pytest.mark.parametrize("p", [0.1, 0.5, 0.999])
def test_values(pk, dtype, rows, H, pad, p):
    g = torch.Generator().manual_seed(H)
    x = torch.randn(rows, H + pad, generator=g).to(dtype)[:, :H]
    r = torch.randn(rows, H, generator=g).to(dtype)
    m, up = kept(rows, H, p, 2)
    y = pk.drop_apply(x.cuda()[:, :H] if not pad else x.cuda(), make(pk, rows, H, p, 2))
    # one product in fp32, one rounding to the type: the same bits
    want = torch.where(m, x.float() * float(up), 0.0)
    assert torch.equal(y.cpu(), want.to(dtype))
    # with the residual: one fp32 addition more, one rounding
    y = pk.drop_apply(x.cuda(), make(pk, rows, H, p, 2), residual=r.cuda())
    exact = want.double() + r.double()
    tol = exact.abs() * (2.0 ** -8 if dtype == BF16 else 0) + 2.0 ** -23 * (want.double().abs() + r.double().abs())
    assert ((y.cpu().double() - exact).abs() <= tol).all()


def test_masks_of_other_keys_and_sites_differ(pk):
    rows, H, p = 64, 1024, 0.5
    x = torch.ones(rows, H, device="cuda")
    base = pk.drop_apply(x, make(pk, rows, H, p)) != 0
    assert abs(float(base.float().mean()) - 0.5) < 5 * 0.5 / (rows * H) ** 0.5
    others = [make(pk, rows, H, p, 1), make(pk, rows, H, p, layer=8), make(pk, rows, H, p, step=1), make(pk, rows, H, p, seed=1),
              make(pk, rows, H, p, microbatch=4), make(pk, rows, H, p, B=2)]
    for d in others:
        same = ((pk.drop_apply(x, d) != 0) == base).float().mean()
        assert abs(float(same) - 0.5) < 5 * 0.5 / (rows * H) ** 0.5
    # nor does it share the boundary's draws of the same fields
    _, bits = pk.ac_bern_mask(rows, H, 0.5, pk.make_key(B=1, S=rows, H=H, **FIELDS))
    word = bits.view(rows, H // 32, 1) >> torch.arange(32, device="cuda", dtype=torch.int32) & 1
    same = (word.view(rows, H).bool() == base).float().mean()
    assert abs(float(same) - 0.5) < 5 * 0.5 / (rows * H) ** 0.5


def test_dropped_places_hold_zero_whatever_was_there(pk):
    rows, H, p = 16, 600, 0.5
    m, _ = kept(rows, H, p, 0)
    for bad in (float("nan"), float("inf"), -float("inf")):
        x = torch.full((rows, H), bad, dtype=BF16, device="cuda")
        y = pk.drop_apply(x, make(pk, rows, H, p)).cpu()
        assert (y[~m] == 0).all() and not torch.signbit(y[~m]).any()
        assert torch.isnan(y[m]).all() if bad != bad else (y[m] == bad).all()


def test_none_dropped_no_rows_and_in_place(pk):
    x = torch.randn(33, 130, device="cuda").bfloat16()
    assert torch.equal(pk.drop_apply(x, make(pk, 33, 130, 0.0)), x)
    e = torch.empty(0, 130, device="cuda")
    assert pk.drop_apply(e, pk.Drop(0.1, pk.make_key(B=0, S=0, H=130, **FIELDS))).shape == (0, 130)
    d, r = make(pk, 33, 130, 0.2), torch.randn(33, 130, device="cuda").bfloat16()
    want = pk.drop_apply(x, d, r)
    a, b = x.clone(), r.clone()
    pk.drop_apply(a, d, r, y=a)
    pk.drop_apply(x, d, b, y=b)
    assert torch.equal(a, want) and torch.equal(b, want)
    # columns behind the last one stay
    wide = torch.full((33, 140), 7.0, dtype=BF16, device="cuda")
    pk.drop_apply(x, d, r, y=wide[:, :130])
    assert torch.equal(wide[:, :130], want) and (wide[:, 130:] == 7).all()


def test_more_than_two_to_the_31_elements(pk):
    rows, H = 70001, 32000
    x = torch.ones(rows, H, dtype=BF16, device="cuda")
    pk.drop_apply(x, make(pk, rows, H, 0.1), y=x)
    m, up = kept(rows, H, 0.1, 0, first=rows - 3, count=3)
    assert torch.equal(x[-3:].cpu(), torch.where(m, torch.tensor(float(up)), 0.0).bfloat16())
    assert abs(float((x[::997] != 0).float().mean()) - 58982 / 65536) < 1e-3


def test_another_stream_and_replays_of_a_graph(pk):
    rows, H = 512, 1024
    x, r, d = torch.randn(rows, H, device="cuda"), torch.randn(rows, H, device="cuda"), make(pk, rows, H, 0.1)
    want = pk.drop_apply(x, d, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = pk.drop_apply(x, d, r, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(y, want)
    out = torch.empty_like(x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pk.drop_apply(x, d, r, y=out)
    for i in range(3):
        x.copy_(torch.randn(rows, H, device="cuda"))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, pk.drop_apply(x, d, r))
