"""Rows that hold NaN where the mask drops every value that it reaches: what lies past the end of a row, in a group of
codes, in a sum over the row, has no say in the values that exist."""
import pytest
import torch

from test_gpu_drop import kept, make
from test_gpu_join import BF16, EPS, F32, SCALE, TOL, near, tensors

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


@pytest.mark.parametrize("H", [130, 1025, 2050, 5121, 9089, 16513])
def test_codes_of_a_last_group_that_is_dropped_whole(pk, H):
    """A NaN of the branch reaches the row's kept values by its norm; a group of which the mask keeps none holds the
    residual alone, and so do its codes."""
    rows, p = 40, 0.9
    t = tensors(rows, H, F32, 0)
    t["b"][:, 0] = NAN
    last = H // 128 * 128
    whole = (~kept(rows, H, p, 3)[0][:, last:]).all(1).cuda()
    assert whole.sum() >= 10
    j = pk.join_forward(t["r"], t["b"], t["post"], t["gate"], None, SCALE, make(pk, rows, H, p, 3), EPS, checkpoint="out")
    assert torch.equal(j.out[whole, last:], SCALE * t["r"][whole, last:])
    want = pk.q8_encode(j.out)
    assert torch.equal(j.q_out.scales[whole, -1], want.scales[whole, -1]) and torch.isfinite(want.scales[whole, -1]).all()
    assert torch.equal(j.q_out.codes[whole, last:], want.codes[whole, last:])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_row_that_is_dropped_whole(pk, dtype):
    """Forward the norm of such a row is the scaled residual's; backward nothing reaches the branch."""
    rows, H, p = 64, 3, 0.9
    t = tensors(rows, H, dtype, 0)
    drop = make(pk, rows, H, p, 3)
    whole = (~kept(rows, H, p, 3)[0]).all(1).cuda()
    assert whole.sum() >= 20
    bad = t["b"].clone()
    bad[:, 0] = NAN
    j = pk.join_forward(t["r"], bad, t["post"], t["gate"], t["pre"], SCALE, drop, EPS)
    r = SCALE * t["r"][whole].double()
    rstd = 1 / (r.square().mean(1) + EPS).sqrt()
    near(j.rstd_pre[whole], rstd, TOL[F32])
    near(j.y[whole], r * rstd[:, None] * t["pre"].double(), TOL[dtype])
    # a gradient that holds NaN, of a branch that does not
    j = pk.join_forward(t["r"], t["b"], t["post"], t["gate"], t["pre"], SCALE, drop, EPS)
    t["dy"][:, 0] = NAN
    d = pk.join_backward(t["dout"], t["dy"], j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE, drop)
    assert (d.db[whole] == 0).all() and torch.isnan(d.dr).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H", [8201, 16391])
def test_a_wide_row_that_is_dropped_whole(pk, dtype, H):
    rows, p = 24, 1 - 2.0 ** -16
    t = tensors(rows, H, dtype, 0)
    drop = make(pk, rows, H, p, 3)
    whole = (~kept(rows, H, p, 3)[0]).all(1).cuda()
    assert 10 <= whole.sum() < rows
    j = pk.join_forward(t["r"], t["b"], t["post"], t["gate"], t["pre"], SCALE, drop, EPS)
    t["dy"][:, 0] = NAN
    d = pk.join_backward(t["dout"], t["dy"], j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE, drop)
    assert (d.db[whole] == 0).all() and torch.isnan(d.dr).all() and torch.isnan(d.db[~whole]).all()


def test_a_source_of_the_other_form_that_is_not_read(pk):
    """A tensor beside a checkpoint, of which the formula reads one: the other has no say."""
    rows, H = 50, 300
    t = tensors(rows, H, F32, 0)
    q = pk.q8_encode(t["b"])
    j = pk.join_forward(t["r"], t["b"], None, None, t["pre"], SCALE, None, EPS)
    want = pk.join_backward(t["dout"], t["dy"], j.out, None, None, j.rstd_pre, pre=t["pre"], scale=SCALE)
    got = pk.join_backward(t["dout"], t["dy"], j.out, q, None, j.rstd_pre, pre=t["pre"], scale=SCALE)
    assert all(torch.equal(a, b) for a, b in zip(got, want) if b is not None)
    want = pk.join_backward(t["dout"], None, None, t["b"], gate=t["gate"], scale=SCALE)
    got = pk.join_backward(t["dout"], None, q, t["b"], gate=t["gate"], scale=SCALE)
    assert all(torch.equal(a, b) for a, b in zip(got, want) if b is not None)
