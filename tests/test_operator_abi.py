"""What the norm, the linear layers and the checkpoints refuse, on the host and
before any HIP call (no GPU needed), and their workspaces' sizes."""
import ctypes as C

import pytest

EINVAL, EDTYPE, EALIGN, ENOSPC = -1, -2, -3, -5
F = 0x10000


@pytest.fixture(scope="module")
def pk():
    import paper_2609_14339_amd as pk
    return pk


def q8(pk, codes=F, scales=F, ldc=1 << 20, lds=1 << 20):
    return C.byref(pk._Q8Tensor(codes, scales, ldc, lds))


def err(pk):
    return pk.lib.acsc_last_error().decode()


def test_checkpoints(pk):
    enc = lambda x=F, dt=1, rows=4, H=300, ld=300, q=None: pk.lib.q8_encode(x, dt, rows, H, ld, q or q8(pk), None)
    assert enc(dt=5) == EDTYPE
    assert enc(rows=-1) == EINVAL and enc(rows=1 << 31) == EINVAL
    assert enc(H=0) == EINVAL and enc(H=(1 << 22) + 1, ld=1 << 23) == EINVAL
    assert enc(ld=299) == EINVAL and "299" in err(pk)
    assert enc(x=None) == EINVAL
    assert enc(x=F + 1) == EALIGN and enc(x=F + 2, dt=0) == EALIGN
    assert enc(q=q8(pk, ldc=299)) == EINVAL and enc(q=q8(pk, lds=2)) == EINVAL
    assert enc(q=q8(pk, codes=None)) == EINVAL and enc(q=q8(pk, scales=F + 2)) == EALIGN
    assert pk.lib.q8_encode(F, 1, 4, 300, 300, None, None) == EINVAL
    assert enc(x=None, rows=0, q=q8(pk, None, None)) == 0
    dec = lambda q=None, act=0, y=F, dt=1, ld=300: pk.lib.q8_decode(q or q8(pk), 4, 300, act, y, dt, ld, None)
    assert dec(act=4) == EINVAL and dec(act=-1) == EINVAL
    assert dec(y=None) == EINVAL and dec(ld=100) == EINVAL and dec(dt=2) == EDTYPE and dec(y=F + 1) == EALIGN


def test_norm(pk):
    def fwd(x=F, dt=1, rows=4, H=64, ldx=64, gamma=F, beta=F, eps=1e-5, y=2 * F, ldy=64, mean=F, rstd=F, q=None):
        return pk.lib.ln_forward(x, dt, rows, H, ldx, gamma, beta, eps, y, ldy, mean, rstd, q, None)
    assert fwd(dt=3) == EDTYPE
    assert fwd(H=0) == EINVAL and fwd(H=32769, ldx=1 << 20, ldy=1 << 20) == EINVAL
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert fwd(eps=eps) == EINVAL
    assert fwd(ldx=63) == EINVAL and fwd(ldy=63) == EINVAL and fwd(x=None) == EINVAL and fwd(y=None) == EINVAL
    assert fwd(gamma=F + 1) == EALIGN and fwd(mean=F + 2) == EALIGN
    assert fwd(x=F, y=F, ldy=72) == EINVAL and "place" in err(pk)
    assert fwd(q=q8(pk, ldc=63)) == EINVAL
    assert fwd(x=None, y=None, rows=0) == 0

    def bwd(dy=F, x=2 * F, q=None, dt=1, rows=4, H=64, mean=F, rstd=F, gamma=F, add=None, ldadd=0, dx=3 * F, lddx=64,
            dg=F, db=F, ws=F, n=1 << 30):
        return pk.lib.ln_backward(dy, 64, x, 64, q, dt, rows, H, mean, rstd, gamma, add, ldadd, dx, lddx, dg, db, 0, ws, n,
                                  None)
    assert bwd(x=None) == EINVAL and bwd(q=q8(pk)) == EINVAL and "exactly one" in err(pk)
    assert bwd(mean=None) == EINVAL and bwd(dy=None) == EINVAL and bwd(dx=None) == EINVAL
    assert bwd(add=F, ldadd=10) == EINVAL and bwd(dx=F, lddx=80) == EINVAL
    assert bwd(ws=None) == EINVAL and bwd(ws=F + 8) == EALIGN and bwd(n=100) == ENOSPC
    assert bwd(dg=F + 1) == EALIGN
    assert bwd(x=None, dy=None, dx=None, dg=None, db=None, rows=0, ws=None, n=0) == 0
    again = lambda x, q: pk.lib.ln_recompute(x, 64, q, 1, 4, 64, F, F, F, F, 2 * F, 64, None)
    assert again(None, None) == EINVAL and again(F, q8(pk)) == EINVAL


def test_linear(pk):
    def fwd(x=F, ldx=64, dt=1, rows=4, n_in=64, n_out=32, W=2 * F, ldw=64, bias=F, act=1, res=None, ldr=0, y=3 * F, ldy=32,
            z=None, ldz=32, q=None, ws=F, n=1 << 30):
        return pk.lib.lin_forward(x, ldx, dt, rows, n_in, n_out, W, ldw, bias, act, res, ldr, y, ldy, z, ldz, q, ws, n, None)
    assert fwd(dt=2) == EDTYPE and fwd(act=9) == EINVAL
    assert fwd(n_in=0) == EINVAL and fwd(n_out=0) == EINVAL and fwd(rows=-1) == EINVAL and fwd(rows=1 << 31) == EINVAL
    assert fwd(ldx=63) == EINVAL and fwd(ldw=63) == EINVAL and fwd(ldy=31) == EINVAL and fwd(res=F, ldr=31) == EINVAL
    assert fwd(x=None) == EINVAL and fwd(W=None) == EINVAL and fwd(y=None) == EINVAL
    assert fwd(x=F + 1) == EALIGN and fwd(bias=F + 1) == EALIGN and fwd(z=F + 1) == EALIGN
    assert fwd(y=F) == EINVAL and fwd(y=2 * F) == EINVAL and "overlap" in err(pk)
    assert fwd(res=3 * F, ldr=40) == EINVAL
    assert fwd(z=F, ldz=31) == EINVAL and fwd(q=q8(pk, lds=0)) == EINVAL
    big = dict(rows=64, n_in=8192, ldx=8192, ldw=8192)
    need = C.c_size_t(0)
    assert pk.lib.lin_workspace_size(0, 64, 8192, 32, 1, C.byref(need)) == 0 and need.value > 0
    assert fwd(**big, n=need.value - 1) == ENOSPC and fwd(**big, ws=None) == EINVAL and fwd(**big, ws=F + 16) == EALIGN
    assert fwd(x=None, W=None, y=None, rows=0) == 0

    def bin_(dz=F, W=2 * F, act=0, z=None, q=None, dx=3 * F, lddx=64, dt=1, ldw=64):
        return pk.lib.lin_backward_input(dz, 32, dt, 4, 64, 32, W, ldw, act, z, 64, q, dx, lddx, F, 1 << 30, None)
    assert bin_(act=2) == EINVAL and bin_(act=2, z=F, q=q8(pk)) == EINVAL and "exactly one" in err(pk)
    assert bin_(dx=F) == EINVAL and bin_(lddx=63) == EINVAL and bin_(ldw=63) == EINVAL and bin_(dt=7) == EDTYPE

    def wgt(dz=F, x=2 * F, q=None, act=0, dt=1, dW=3 * F, dw_dt=1, lddw=64, db=F, acc=0, ws=F, n=1 << 30, rows=4):
        return pk.lib.lin_backward_weight(dz, 32, x, 64, q, act, dt, rows, 64, 32, dW, dw_dt, lddw, db, acc, ws, n, None)
    assert wgt(dw_dt=4) == EDTYPE and wgt(dt=4) == EDTYPE and wgt(act=7) == EINVAL
    assert wgt(x=None) == EINVAL and wgt(q=q8(pk)) == EINVAL and wgt(dW=None) == EINVAL and wgt(lddw=63) == EINVAL
    assert wgt(dW=3 * F + 2, dw_dt=0) == EALIGN and wgt(db=F + 1) == EALIGN
    assert wgt(n=10, act=2, rows=100) == ENOSPC and wgt(n=1 << 30, act=2, ws=F + 16, rows=100) == EALIGN
    assert pk.lib.lin_workspace_size_unaligned(2, 100, 64, 32, 1, C.byref(need)) == 0 and need.value > 0
    assert wgt(dz=F + 2, n=64, rows=100) == ENOSPC       # an unaligned operand is copied first
    assert wgt(dz=None, x=None, rows=0, acc=1) == 0
    assert pk.lib.lin_backward_act(F, 32, None, 32, None, 1, 4, 32, 2, F, 32, None) == EINVAL
    assert pk.lib.lin_backward_act(F, 32, F, 32, None, 1, 4, 32, 2, F, 40, None) == EINVAL


def test_workspace_sizes(pk):
    b = C.c_size_t(0)
    for op in (0, 1, 2):
        assert pk.lib.lin_workspace_size(op, 0, 64, 64, 1, C.byref(b)) == 0 and b.value == 0
        assert pk.lib.lin_workspace_size(op, 4, 0, 64, 1, C.byref(b)) == EINVAL
        assert pk.lib.lin_workspace_size(op, 4, 64, 64, 1, None) == EINVAL
    assert pk.lib.lin_workspace_size(3, 4, 64, 64, 1, C.byref(b)) == EINVAL
    assert pk.lib.ln_workspace_size(16384, 8192, C.byref(b)) == 0 and b.value <= 64 << 20
    assert pk.lib.ln_workspace_size(4, 40000, C.byref(b)) == EINVAL


def test_binding_refuses(pk):
    import torch
    x, W = torch.zeros(4, 8), torch.zeros(6, 8)
    for call in (lambda: pk.lin_forward(x, W), lambda: pk.ln_forward(x), lambda: pk.q8_encode(x),
                 lambda: pk.lin_backward_weight(x, x)):
        with pytest.raises(pk.AcscError, match="GPU"):
            call()
    with pytest.raises(pk.AcscError, match="2-D"):
        pk.ln_forward(torch.zeros(3))
    with pytest.raises(pk.AcscError, match="activation"):
        pk._act("tanh")
