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
