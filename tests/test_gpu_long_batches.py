"""Row counts whose launches need more threads than a grid has along x (2^32), and more than 2^31 elements."""
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


# a row of up to 1024 columns is a quarter of a workgroup of 256 threads, a wider one a workgroup
@pytest.mark.parametrize("rows,H", [((1 << 26) + 5, 3), ((1 << 24) + 3, 1032)])
def test_norm_of_many_rows(pk, rows, H):
    x = torch.zeros(rows, H, dtype=BF16, device="cuda")
    g = torch.Generator().manual_seed(1)
    gamma, beta = torch.randn(H, generator=g).to(BF16).cuda(), torch.randn(H, generator=g).to(BF16).cuda()
    # rows at both ends and about where the grid goes on
    at = torch.cat([torch.arange(k - 9, k + 9) for k in (9, 1 << 20, 1 << 22, rows - 9)] +
                   [torch.arange(k - 4, k) for k in (1 << 24, 1 << 26) if k <= rows]).cuda()
    x[at] = torch.randn(len(at), H, generator=g).to(BF16).cuda()
    want = pk.ln_forward(x[at], gamma, beta)
    y, mean, rstd, _ = pk.ln_forward(x, gamma, beta)
    assert torch.equal(y[at], want[0]) and torch.equal(mean[at], want[1]) and torch.equal(rstd[at], want[2])
    # the rows of zeros between them give beta
    step = max(1, rows // 4099)
    between = torch.arange(0, rows, step, device="cuda")
    between = between[~torch.isin(between, at)]
    assert torch.equal(y[between], beta.expand(len(between), H))
    del y
    assert torch.equal(pk.ln_recompute(x, mean, rstd, gamma, beta)[at], want[0])
