"""What the gated block's gradients take as sources, on the host and before any HIP call (no GPU needed)."""
import ctypes as C

import pytest

EINVAL = -1
F = 0x10000


@pytest.fixture(scope="module")
def pk():
    import paper_2609_14339_amd as pk
    return pk


def test_a_source_that_is_not_read_may_be_of_either_form(pk):
    """out is read with dy, b with post or gate; the two are of one form where both are read, and only there."""
    q = C.byref(pk._Q8Tensor(F, F, 64, 1))

    def call(dy=None, out=None, qo=None, b=None, qb=None, gate=None):
        return pk.lib.join_backward(F, 64, dy, 64, out, 64, qo, b, 64, qb, 1, 0, 64, None, gate, 1.0, None, None, None, F, 5 * F, 64,
                                    6 * F, 64, None, None, None, 0, None, 0, None)
    assert call(dy=2 * F, out=3 * F, qb=q) == 0 and call(dy=2 * F, qo=q, b=4 * F) == 0        # b is not read
    assert call(out=3 * F, qb=q, gate=F) == 0 and call(qo=q, b=4 * F, gate=F) == 0            # out is not
    assert call(dy=2 * F, out=3 * F, b=4 * F, gate=F) == 0 and call(dy=2 * F, qo=q, qb=q, gate=F) == 0
    for mixed in (dict(out=3 * F, qb=q), dict(qo=q, b=4 * F)):
        assert call(dy=2 * F, gate=F, **mixed) == EINVAL
        assert "both" in pk.lib.acsc_last_error().decode()


def test_the_bias_gradient_of_a_given_gradient(pk):
    EALIGN, ENOSPC = -3, -5
    q = C.byref(pk._Q8Tensor(F, F, 32, 1))

    def call(dh=F, z=2 * F, qg=None, qu=None, dt=1, rows=40, a=3, dz=3 * F, lddz=64, h=None, ldh=32, ldz=64, db=4 * F, ws=5 * F,
             n=1 << 30, acc=0, Fh=32):
        return pk.lib.glu_backward_act_bias(dh, 32, z, ldz, qg, qu, dt, rows, Fh, a, dz, lddz, h, ldh, db, acc, ws, n, None)
    assert call(db=None) == EINVAL and call(db=4 * F + 2) == EALIGN
    assert call(ws=None) == EINVAL and call(ws=5 * F + 16) == EALIGN and call(n=255) == ENOSPC
    assert call(z=None) == EINVAL and call(qg=q, qu=q) == EINVAL and call(z=None, qg=q) == EINVAL
    assert call(dh=None) == EINVAL and call(dz=None) == EINVAL and call(lddz=63) == EINVAL and call(ldz=63) == EINVAL
    assert call(dz=F) == EINVAL and call(dz=2 * F, lddz=80) == EINVAL and call(h=2 * F) == EINVAL and call(h=F, ldh=40) == EINVAL
    assert call(a=4) == EINVAL and call(dt=3) == -2 and call(h=3 * F) == EINVAL and call(rows=-1) == EINVAL and call(Fh=0) == EINVAL
    assert call(dh=None, z=None, dz=None, rows=0, acc=1, ws=None, n=0) == 0
    b = C.c_size_t(0)
    assert pk.lib.glu_bias_workspace_size(0, 32, C.byref(b)) == 0 and b.value == 0
    assert pk.lib.glu_bias_workspace_size(4, 32, None) == EINVAL and pk.lib.glu_bias_workspace_size(4, 0, C.byref(b)) == EINVAL
    for rows, Fh, parts in ((1, 1, 0), (16, 4096, 0), (16384, 8192, 1), ((1 << 31) - 1, 1 << 21, 0), (1 << 30, 512, 1), (1 << 30, 513, 1)):
        assert pk.lib.glu_bias_workspace_size(rows, Fh, C.byref(b)) == 0 and b.value <= 32 << 20 and (b.value > 0) == bool(parts)


def test_coded_products_take_a_bounded_workspace(pk):
    """Where a product's tiles hold no whole groups its pre-activations go through the workspace, a part of them at a time:
    256 MiB at most, however many rows there are, or one row of tiles (of 128 rows of 2 F fp32 values at most)."""
    import torch
    for rows, n_in, Fh in ((16384, 2048, 8192), (4096, 4096, 14336), (1 << 20, 64, 1024), (65536, 33, 100), (300, 64, 1 << 20)):
        for dt in (torch.float32, torch.bfloat16):
            most = max(256 << 20, 128 * 4 * 2 * (Fh + 64)) + (1 << 20)
            copies = dt.itemsize * ((rows + 2 * Fh) * (n_in + 8))
            assert pk.glu_workspace_size(pk.GLU_FORWARD, rows, n_in, Fh, dt, True) <= most + (copies if n_in % 2 else 0)
            assert pk.glu_workspace_size_unaligned(pk.GLU_FORWARD, rows, n_in, Fh, dt, True) <= most + copies
