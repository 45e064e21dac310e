"""8-bit activation checkpoints against their definition: codes and scales bit
for bit, values of them exactly, activations within the arithmetic of one
fp32 evaluation and one rounding."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
GROUP = 128


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def reference(x):
    """Codes and scales of x (CPU fp32), operation by operation."""
    rows, H = x.shape
    n = -(-H // GROUP)
    v = torch.zeros(rows, n * GROUP)
    v[:, :H] = x.float()
    v = v.view(rows, n, GROUP)
    a = v.abs().amax(2)                       # NaN propagates
    bad = ~torch.isfinite(a)
    small = a < 2.0 ** -120
    scale = torch.where(bad, float("nan"), torch.where(small, 0.0, a / torch.full_like(a, 127)))
    # quotients of tensors: torch takes 127 / a as 127 times a's reciprocal, which is rounded twice
    inv = torch.where(bad | small, 0.0, torch.full_like(a, 127) / a)
    codes = torch.round(torch.where((bad | small)[..., None], 0.0, v * inv[..., None]))
    return codes.reshape(rows, -1)[:, :H].to(torch.int8), scale


def draw(rows, H, dtype, pad, seed=0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, H + pad, generator=g) * torch.exp(torch.randn(rows, H + pad, generator=g) * 2)
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,H,pad", [(1, 1, 0), (1, 128, 0), (3, 7, 0), (2, 129, 3), (5, 1023, 2), (64, 2048, 0),
                                        (7, 513, 8), (130, 4097, 5), (1, 28672, 0)])
def test_codes_and_scales_equal_the_definition(pk, dtype, rows, H, pad):
    x = draw(rows, H, dtype, pad, seed=H)
    q = pk.q8_encode(x.cuda()[:, :H])
    codes, scales = reference(x[:, :H])
    assert torch.equal(q.codes.cpu(), codes)
    assert torch.equal(q.scales.cpu(), scales)
    # reading back: the product of code and scale, rounded once
    y = pk.q8_decode(q, dtype)
    want = (codes.float() * scales.repeat_interleave(GROUP, 1)[:, :H]).to(dtype)
    assert torch.equal(y.cpu(), want)
    # what the format promises: half a step
    step = scales.repeat_interleave(GROUP, 1)[:, :H].double()
    assert ((codes.double() * step - x[:, :H].double()).abs() <= step * (0.5 + 127 * 2.0 ** -22)).all()


def test_zeros_tiny_infinite_and_nan_groups(pk):
    x = torch.randn(8, 5 * GROUP + 9)
    x[0, :GROUP] = 0
    x[1, GROUP:2 * GROUP] = 1e-40                       # below 2^-120
    x[2, 3 * GROUP + 5] = float("inf")
    x[3, 5] = float("-inf")
    x[4, 2 * GROUP + 77] = float("nan")
    x[5, 5 * GROUP + 8] = float("nan")                  # the last, partial group
    x[6, :GROUP] = 2.0 ** -120                          # the smallest that is kept
    x[7, :GROUP] = 3.4e38                               # the largest
    q = pk.q8_encode(x.cuda())
    codes, scales = reference(x)
    assert torch.equal(q.codes.cpu(), codes)
    assert torch.equal(q.scales.cpu().nan_to_num(-1.0), scales.nan_to_num(-1.0))
    y = pk.q8_decode(q, torch.float32).cpu()
    assert torch.isnan(y).sum() == 3 * GROUP + 9
    assert (y[0, :GROUP] == 0).all() and (y[1, GROUP:2 * GROUP] == 0).all()
    assert torch.isfinite(y[6]).all() and torch.isfinite(y[7]).all() and (y[6, :GROUP] > 0).all()


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_reading_back_through_an_activation(pk, act, dtype):
    x = draw(33, 700, torch.float32, 0, seed=5)
    x[0, :4] = torch.tensor([-100.0, -12.0, 100.0, 0.0])
    q = pk.q8_encode(x.cuda())
    y = pk.q8_decode(q, dtype, act=act).cpu().double()
    z = (q.codes.float() * q.scales.repeat_interleave(GROUP, 1)[:, :700]).cpu().double()
    ref = {"relu": lambda: z.clamp_min(0), "gelu": lambda: z * 0.5 * torch.erfc(-z / math.sqrt(2)),
           "silu": lambda: z * torch.sigmoid(z)}[act]()
    # Phi(z) or sigmoid(z) within 4 units of 2^-24 of 1, times |z|; then the rounding of y
    tol = 4 * 2.0 ** -24 * z.abs() + ref.abs() * (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -22)
    assert ((y - ref).abs() <= tol + 1e-38).all()


def test_no_rows(pk):
    q = pk.q8_encode(torch.empty(0, 300, device="cuda"))
    assert q.codes.shape == (0, 300) and q.scales.shape == (0, 3)
    assert pk.q8_decode(q, torch.bfloat16).shape == (0, 300)


def test_only_the_tensor_is_written(pk):
    """Columns past H of a wider output, codes and scales keep their bytes."""
    rows, H = 9, 200
    x = draw(rows, H, torch.bfloat16, 0).cuda()
    codes = torch.full((rows, H + 13), 99, dtype=torch.int8, device="cuda")
    scales = torch.full((rows, 5), -3.0, device="cuda")
    q = pk.q8_encode(x, q=pk.Q8(codes[:, :H], scales[:, :2]))
    wide = torch.full((rows, H + 3), 7.0, dtype=torch.bfloat16, device="cuda")
    pk.q8_decode(q, torch.bfloat16, y=wide[:, :H])
    assert (codes[:, H:] == 99).all() and (scales[:, 2:] == -3).all() and (wide[:, H:] == 7).all()
    assert torch.equal(wide[:, :H], pk.q8_decode(pk.q8_encode(x), torch.bfloat16))


def test_row_offsets_past_32_bits(pk):
    ld = (1 << 31) + 264
    buf = torch.empty(2 * ld + 256, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(buf, (3, 256), (ld, 1))
    src = draw(3, 256, torch.bfloat16, 0, seed=3).cuda()
    x.copy_(src)
    q = pk.q8_encode(x)
    want = pk.q8_encode(src)
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
