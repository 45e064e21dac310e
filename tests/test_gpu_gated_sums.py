"""Gradients of the gains over more than 2^31 elements and more than 2^20 workgroups' rows: gradients that are zero but in
some rows, so that a row that is lost, or counted twice, shows in the sums of few terms."""
import pytest
import torch

from test_gpu_drop import make
from test_gpu_gated_limits import gauss
from test_gpu_join import BF16, EPS, SCALE, U, ref_backward

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    yield pk
    torch.cuda.empty_cache()


def some_rows(rows, H):
    """The first and last rows, those beside element 2^31 and row 2^20 and 2^22, and one in each of 200 equal runs."""
    g = torch.Generator().manual_seed(rows)
    at = {0, 1, 2, 3, 4, rows - 1, rows - 2, rows - 3, rows - 4, rows - 5}
    for border in (2 ** 31 // H, 2 ** 20, 2 ** 22):
        at |= {r for r in range(border - 2, border + 3) if r < rows}
    run = rows // 200
    at |= {i * run + int(torch.randint(run, (1,), generator=g)) for i in range(200)}
    return torch.tensor(sorted(at), device="cuda")


@pytest.mark.parametrize("rows,H", [(70001, 32000), (300001, 8000), (1200003, 2000), (1200003, 1100), (5000003, 64)])
def test_sums_over_every_row(pk, rows, H):
    at = some_rows(rows, H)
    r, b = gauss(rows, H, BF16, 1), gauss(rows, H, BF16, 2)
    gains = {k: (torch.randn(H, generator=torch.Generator("cuda").manual_seed(9 + i), device="cuda") * 0.2 + 1).bfloat16()
             for i, k in enumerate(("post", "gate", "pre"))}
    drop = make(pk, rows, H, 0.1, 3)
    up = 65536 / 58982      # the threshold floor(0.9 * 65536 + 1/2)
    j = pk.join_forward(r, b, gains["post"], gains["gate"], gains["pre"], SCALE, drop, EPS)
    ones = r.fill_(1.0)
    factor = (pk.drop_apply(ones, drop, y=ones)[at] != 0).double() * up
    del r, ones
    some = {k: gauss(len(at), H, BF16, i) for i, k in enumerate(("dout", "dy"), 3)}
    dout, dy = torch.zeros(rows, H, dtype=BF16, device="cuda"), torch.zeros(rows, H, dtype=BF16, device="cuda")
    dout[at], dy[at] = some["dout"], some["dy"]
    x, kept_b = j.out[at], b[at]
    d = pk.join_backward(dout, dy, j.out, b, j.rstd_post, j.rstd_pre, gains["post"], gains["gate"], gains["pre"], SCALE, drop,
                         dr=dout, db=dy)
    want, size = ref_backward({**some, **gains}, x, kept_b, j.rstd_post[at], j.rstd_pre[at], True, True, True, factor)
    # zeros add nothing to the error: at most len(at) terms and 100 levels of joining, each term within 100 units as in
    # the tests of small sizes
    for name in ("dpost", "dgate", "dpre"):
        got, tol = getattr(d, name).double(), U * (len(at) + 200) * size[name]
        assert torch.isfinite(got).all() and ((got - want[name]).abs() <= tol).all(), name
        # a single row more or less would show: every row has a term of many times the bound
        assert tol.max() < 0.2
    for v in (d.dr, d.db):
        assert torch.equal(v.abs().amax(1).nonzero()[:, 0], at)
