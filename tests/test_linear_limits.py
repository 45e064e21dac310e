"""Linear layers at the largest row counts that they take, from the host side: sizes of workspaces (no GPU needed)."""
import ctypes as C

import pytest

F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def pk():
    import paper_2609_14339_amd as pk
    return pk


def up(n, k):
    return -(-n // k) * k


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("n_in,n_out", [(1, 1), (8, 300), (64, 512), (72, 1300)])
@pytest.mark.parametrize("short", [1, 2, 31, 32, 33, 63, 64, 65, 4096, (1 << 22) - 3, 1 << 22, (1 << 22) + 5, 1 << 23])
def test_weight_gradient_of_nearly_2_31_rows(pk, dt, n_in, n_out, short):
    """db's sums are cut into slices of the rows whatever their number, and the product as it is at half as many rows:
    what is left of the size beside db, the recomputed activation and copies."""
    def pieces(rows):
        b = C.c_size_t(0)
        assert pk.lib.lin_workspace_size(pk.LIN_BACKWARD_WEIGHT, rows, n_in, n_out, dt, C.byref(b)) == 0
        slices = max(1, min(512 // -(-n_out // 512), rows // 32))
        slices = -(-rows // -(-rows // slices))
        es = 2 if dt == BF16 else 4
        recomputed = up(rows * up(n_in, 8) * es, 256)
        copies = sum(up(rows * up(n, 8) * es, 256) for n in (n_in, n_out) if n < 16 // es or n * es % 4)
        return b.value - recomputed - copies - up(slices * n_out * 4, 256)

    assert pieces((1 << 31) - short) == pieces(1 << 30) >= 0


EINVAL = -1


@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("op", [0, 1])
def test_products_of_more_threads_than_a_launch_has(pk, op, dt):
    """256 threads to 128 rows: 2^24 tiles are one too many, and said so before anything is launched."""
    b = C.c_size_t(7)
    for size in (pk.lib.lin_workspace_size, pk.lib.lin_workspace_size_unaligned):
        assert size(op, (1 << 31) - 128, 8, 8, dt, C.byref(b)) == 0
        assert size(op, (1 << 31) - 127, 8, 8, dt, C.byref(b)) == EINVAL and b"too large" in pk.lib.acsc_last_error()
        assert size(op, 1 << 30, 1 << 22, 1 << 22, dt, C.byref(b)) == EINVAL and b.value == 0
    assert pk.lib.lin_workspace_size(2, 100, 1 << 22, 1 << 22, dt, C.byref(b)) == EINVAL
    W = 0x10000
    call = (lambda rows: pk.lib.lin_forward(W, 8, dt, rows, 8, 8, 2 * W, 8, None, 0, None, 0, 3 * W, 8, None, 8, None, W,
                                            1 << 62, None)) if op == 0 else \
        (lambda rows: pk.lib.lin_backward_input(W, 8, dt, rows, 8, 8, 2 * W, 8, 0, None, 8, None, 3 * W, 8, W, 1 << 62, None))
    assert call((1 << 31) - 1) == EINVAL and b"too large" in pk.lib.acsc_last_error()


def test_outputs_in_the_place_of_inputs(pk):
    """What a product still reads while it writes is refused; element by element, a place is taken with its row stride."""
    F, n = 0x10000, 1 << 30
    lin = lambda z, ldz=64: pk.lib.lin_forward(F, 64, 1, 40, 64, 64, 2 * F, 64, None, 1, None, 0, 3 * F, 64, z, ldz, None, F, n,
                                               None)
    assert lin(F) == EINVAL and lin(2 * F) == EINVAL and b"z must not overlap" in pk.lib.acsc_last_error()
    dx = lambda at, ld: pk.lib.lin_backward_input(F, 64, 1, 40, 64, 64, 2 * F, 64, 2, 4 * F, 64, None, at, ld, F, n, None)
    assert dx(4 * F, 72) == EINVAL and b"place of z" in pk.lib.acsc_last_error()
    dw = lambda at: pk.lib.lin_backward_weight(F, 64, 2 * F, 64, None, 0, 1, 64, 64, 64, at, 1, 64, None, 0, F, n, None)
    assert dw(F) == EINVAL and dw(2 * F) == EINVAL and b"overlap" in pk.lib.acsc_last_error()
    assert pk.lib.lin_backward_act(F, 64, 2 * F, 64, None, 1, 40, 64, 2, 2 * F, 72, None) == EINVAL
    assert pk.lib.ln_backward(F, 64, 2 * F, 64, None, 1, 40, 64, F, F, F, None, 0, 2 * F, 72, None, None, 0, None, 0,
                              None) == EINVAL and b"place of x" in pk.lib.acsc_last_error()
