"""What dropout, the joined norms and the gated layer refuse, on the host and before any HIP call (no GPU needed), and
their workspaces' sizes and plans."""
import ctypes as C

import pytest
import torch

EINVAL, EDTYPE, EALIGN, ENOSPC = -1, -2, -3, -5
F = 0x10000


@pytest.fixture(scope="module")
def pk():
    import paper_2609_14339_amd as pk
    return pk


def q8(pk, codes=F, scales=F, ldc=1 << 22, lds=1 << 20):
    return C.byref(pk._Q8Tensor(codes, scales, ldc, lds))


def drop(pk, rows=4, H=64, p=0.1, B=2):
    return C.byref(pk._DropMask(pk.make_key(seed=1, layer=0, step=0, microbatch=0, B=B, S=rows // B, H=H), 0, p))


def err(pk):
    return pk.lib.acsc_last_error().decode()


def test_drop(pk):
    def call(x=F, dt=1, rows=4, H=64, ldx=64, d=0, res=None, ldr=64, y=2 * F, ldy=64):
        return pk.lib.drop_apply(x, dt, rows, H, ldx, drop(pk) if d == 0 else d, res, ldr, y, ldy, None)
    assert call(dt=4) == EDTYPE and call(rows=-1) == EINVAL and call(rows=1 << 31) == EINVAL and call(H=0) == EINVAL
    assert call(d=None) == EINVAL
    for p in (-0.1, 1.0, 1.5, float("nan"), 1 - 2.0 ** -18):
        assert call(d=drop(pk, p=p)) == EINVAL
    assert call(d=drop(pk, H=65)) == EINVAL and call(d=drop(pk, rows=6)) == EINVAL and "key" in err(pk)
    assert call(x=None) == EINVAL and call(y=None) == EINVAL and call(ldx=63) == EINVAL and call(ldy=63) == EINVAL
    assert call(x=F + 1) == EALIGN and call(res=F + 1) == EALIGN and call(res=F, ldr=63) == EINVAL
    assert call(y=F, ldy=72) == EINVAL and call(res=2 * F, ldr=72) == EINVAL and "place" in err(pk)
    assert call(x=None, y=None, rows=0, d=drop(pk, rows=0)) == 0


def test_rms(pk):
    def fwd(x=F, dt=1, rows=4, H=64, ldx=64, gamma=F, eps=1e-5, y=2 * F, ldy=64, rstd=F, q=None):
        return pk.lib.rms_forward(x, dt, rows, H, ldx, gamma, eps, y, ldy, rstd, q, None)
    assert fwd(dt=3) == EDTYPE and fwd(H=0) == EINVAL and fwd(H=32769, ldx=1 << 20, ldy=1 << 20) == EINVAL
    for eps in (0.0, -1.0, float("inf"), float("nan")):
        assert fwd(eps=eps) == EINVAL
    assert fwd(ldx=63) == EINVAL and fwd(ldy=63) == EINVAL and fwd(x=None) == EINVAL and fwd(y=None) == EINVAL
    assert fwd(gamma=F + 1) == EALIGN and fwd(rstd=F + 2) == EALIGN and fwd(x=F, y=F, ldy=72) == EINVAL
    assert fwd(q=q8(pk, ldc=63)) == EINVAL and fwd(x=None, y=None, rows=0) == 0
    again = lambda x, q, r=F: pk.lib.rms_recompute(x, 64, q, 1, 4, 64, r, F, 2 * F, 64, None)
    assert again(None, None) == EINVAL and again(F, q8(pk)) == EINVAL and again(F, None, None) == EINVAL

    def bwd(dy=F, x=2 * F, q=None, dt=1, rows=4, rstd=F, gamma=F, add=None, ldadd=0, dx=3 * F, lddx=64, dg=F, ws=F, n=1 << 30):
        return pk.lib.rms_backward(dy, 64, x, 64, q, dt, rows, 64, rstd, gamma, add, ldadd, dx, lddx, dg, 0, ws, n, None)
    assert bwd(x=None) == EINVAL and bwd(q=q8(pk)) == EINVAL and "exactly one" in err(pk)
    assert bwd(rstd=None) == EINVAL and bwd(dy=None) == EINVAL and bwd(dx=None) == EINVAL
    assert bwd(add=F, ldadd=10) == EINVAL and bwd(dx=F, lddx=80) == EINVAL
    assert bwd(ws=None) == EINVAL and bwd(ws=F + 8) == EALIGN and bwd(n=100) == ENOSPC and bwd(dg=F + 1) == EALIGN
    assert bwd(x=None, dy=None, dx=None, dg=None, rows=0, ws=None, n=0) == 0


def test_join(pk):
    def fwd(r=F, b=2 * F, ldb=64, dt=1, rows=4, H=64, post=F, gate=F, scale=1.0, d=None, pre=F, eps=1e-5, out=3 * F, ldo=64,
            y=4 * F, ldy=64, rp=F, rn=F, qo=None, qb=None):
        return pk.lib.join_forward(r, 64, b, ldb, dt, rows, H, post, gate, scale, d, pre, eps, out, ldo, y, ldy, rp, rn, qo, qb,
                                   None)
    assert fwd(dt=2) == EDTYPE and fwd(H=0) == EINVAL and fwd(rows=-1) == EINVAL and fwd(eps=0.0) == EINVAL
    assert fwd(scale=float("inf")) == EINVAL and fwd(scale=float("nan")) == EINVAL
    assert fwd(r=None) == EINVAL and fwd(b=None) == EINVAL and fwd(out=None) == EINVAL and fwd(ldb=63) == EINVAL
    assert fwd(d=drop(pk, p=1.0)) == EINVAL and fwd(d=drop(pk, H=32)) == EINVAL and fwd(d=drop(pk, rows=8)) == EINVAL
    assert fwd(out=F, ldo=72) == EINVAL and fwd(y=2 * F, ldy=72) == EINVAL and fwd(y=3 * F) == EINVAL
    assert fwd(y=None) == EINVAL and fwd(y=None, pre=None, rn=F) == EINVAL and fwd(post=None) == EINVAL
    assert fwd(post=F + 1) == EALIGN and fwd(gate=F + 1) == EALIGN and fwd(pre=F + 1) == EALIGN and fwd(rn=F + 1) == EALIGN
    assert fwd(qo=q8(pk, ldc=3)) == EINVAL and fwd(qb=q8(pk, lds=0)) == EINVAL
    assert fwd(r=None, b=None, out=None, y=None, rows=0) == 0

    def bwd(dout=F, dy=2 * F, out=3 * F, qo=None, b=4 * F, qb=None, dt=1, rows=4, post=F, gate=F, scale=1.0, d=None, pre=F, rp=F,
            rn=F, dr=5 * F, db=6 * F, lddb=64, dp=F, dg=F, dn=F, ws=F, n=1 << 30):
        return pk.lib.join_backward(dout, 64, dy, 64, out, 64, qo, b, 64, qb, dt, rows, 64, post, gate, scale, d, pre, rp, rn, dr,
                                    64, db, lddb, dp, dg, dn, 0, ws, n, None)
    assert bwd(dt=2) == EDTYPE and bwd(dout=None, dy=None) == EINVAL and bwd(db=None) == EINVAL and bwd(lddb=63) == EINVAL
    assert bwd(out=None) == EINVAL and bwd(b=None) == EINVAL and bwd(qo=q8(pk)) == EINVAL and bwd(qb=q8(pk)) == EINVAL
    assert bwd(b=None, qb=q8(pk)) == EINVAL and "both" in err(pk)
    assert bwd(out=None, qo=q8(pk)) == EINVAL
    assert bwd(rp=None) == EINVAL and bwd(rn=None) == EINVAL and bwd(dy=None) == EINVAL and bwd(post=None) == EINVAL
    assert bwd(gate=None) == EINVAL and bwd(dr=6 * F) == EINVAL and bwd(db=F, lddb=72) == EINVAL
    assert bwd(ws=None) == EINVAL and bwd(ws=F + 8) == EALIGN and bwd(n=100) == ENOSPC and bwd(dn=F + 1) == EALIGN
    assert bwd(scale=float("nan")) == EINVAL and bwd(d=drop(pk, H=32)) == EINVAL
    b = C.c_size_t(0)
    assert pk.lib.join_workspace_size(16384, 8192, C.byref(b)) == 0 and 0 < b.value <= 64 << 20
    assert pk.lib.join_workspace_size(4, 40000, C.byref(b)) == EINVAL and pk.lib.join_workspace_size(4, 64, None) == EINVAL


def test_glu(pk):
    def fwd(x=F, ldx=64, dt=1, rows=4, n_in=64, Fh=32, W=2 * F, ldw=64, bias=F, act=3, h=3 * F, ldh=32, z=None, ldz=64, qg=None,
            qu=None, ws=F, n=1 << 30):
        return pk.lib.glu_forward(x, ldx, dt, rows, n_in, Fh, W, ldw, bias, act, h, ldh, z, ldz, qg, qu, ws, n, None)
    assert fwd(dt=2) == EDTYPE and fwd(act=9) == EINVAL and fwd(n_in=0) == EINVAL and fwd(Fh=0) == EINVAL
    assert fwd(Fh=(1 << 21) + 1, ldh=1 << 22) == EINVAL and fwd(rows=-1) == EINVAL and fwd(rows=1 << 31) == EINVAL
    assert fwd(ldx=63) == EINVAL and fwd(ldw=63) == EINVAL and fwd(ldh=31) == EINVAL and fwd(z=4 * F, ldz=63) == EINVAL
    assert fwd(x=None) == EINVAL and fwd(W=None) == EINVAL and fwd(h=None) == EINVAL
    assert fwd(x=F + 1) == EALIGN and fwd(bias=F + 1) == EALIGN and fwd(z=F + 1) == EALIGN
    assert fwd(h=F) == EINVAL and fwd(h=2 * F) == EINVAL and fwd(z=F) == EINVAL and fwd(z=3 * F) == EINVAL and "overlap" in err(pk)
    assert fwd(qg=q8(pk)) == EINVAL and fwd(qg=q8(pk), qu=q8(pk, lds=0)) == EINVAL
    assert fwd(x=None, W=None, h=None, rows=0) == 0
    need = C.c_size_t(0)
    assert pk.lib.glu_workspace_size(0, 64, 8192, 32, 1, 0, C.byref(need)) == 0 and need.value > 0
    big = dict(rows=64, n_in=8192, ldx=8192, ldw=8192)
    assert fwd(**big, n=need.value - 1) == ENOSPC and fwd(**big, ws=None) == EINVAL and fwd(**big, ws=F + 16) == EALIGN

    def act(dh=F, z=2 * F, qg=None, qu=None, dt=1, a=3, dz=3 * F, lddz=64, h=None, ldh=32, ldz=64):
        return pk.lib.glu_backward_act(dh, 32, z, ldz, qg, qu, dt, 4, 32, a, dz, lddz, h, ldh, None)
    assert act(z=None) == EINVAL and act(qg=q8(pk), qu=q8(pk)) == EINVAL and act(z=None, qg=q8(pk)) == EINVAL
    assert act(dh=None) == EINVAL and act(dz=None) == EINVAL and act(lddz=63) == EINVAL and act(ldz=63) == EINVAL
    assert act(dz=F) == EINVAL and act(dz=2 * F, lddz=80) == EINVAL and act(h=2 * F) == EINVAL and act(h=F, ldh=40) == EINVAL
    assert act(a=4) == EINVAL and act(dt=3) == EDTYPE and act(h=3 * F) == EINVAL

    def inp(dy=F, W=2 * F, z=3 * F, qg=None, qu=None, dz=4 * F, lddz=64, h=None, dt=1, ws=F, ldw=32, db=None, n=1 << 30):
        return pk.lib.glu_backward_input(dy, 64, dt, 4, 32, 64, W, ldw, 3, z, 64, qg, qu, dz, lddz, h, 32, db, 0, ws, n, None)
    assert inp(z=None) == EINVAL and inp(z=None, qu=q8(pk)) == EINVAL and inp(dy=None) == EINVAL and inp(W=None) == EINVAL
    assert inp(dz=F) == EINVAL and inp(dz=2 * F) == EINVAL and inp(h=4 * F) == EINVAL and inp(h=3 * F) == EINVAL
    assert inp(dz=3 * F, lddz=80) == EINVAL and inp(ldw=31) == EINVAL and inp(dt=5) == EDTYPE
    assert inp(db=F + 1) == EALIGN and inp(db=F, n=0) == ENOSPC and inp(db=F, ws=None) == EINVAL


def test_plans_and_workspaces(pk):
    b = C.c_size_t(0)
    for op in (0, 1):
        assert pk.lib.glu_workspace_size(op, 0, 64, 64, 1, 0, C.byref(b)) == 0 and b.value == 0
        assert pk.lib.glu_workspace_size(op, 4, 0, 64, 1, 0, C.byref(b)) == EINVAL
        assert pk.lib.glu_workspace_size(op, 4, 64, 64, 1, 0, None) == EINVAL
        assert pk.lib.glu_workspace_size_unaligned(op, 40, 65, 63, 1, 0, C.byref(b)) == 0 and b.value > 0
    assert pk.lib.glu_workspace_size(2, 4, 64, 64, 1, 0, C.byref(b)) == EINVAL
    # launches of 2^32 threads and more: of tiles, and of the sum that a checkpoint's narrow tiles go through
    for dt, rows, Fh, extra in ((1, 1 << 30, 1 << 20, 0), (1, 1 << 30, 1 << 20, 1), (0, 1 << 26, 1 << 10, 1)):
        assert pk.lib.glu_workspace_size(0, rows, 64, Fh, dt, extra, C.byref(b)) == EINVAL and "too large" in err(pk)
    assert pk.lib.glu_workspace_size(0, 1 << 26, 64, 1 << 10, 0, 0, C.byref(b)) == 0
    bf, f32 = torch.bfloat16, torch.float32
    assert pk.glu_product_plan(0, 1, 4096, 14336, bf)[:2] == (0, 0)
    for rows, n_in, Fh, dt in ((8192, 8192, 28672, bf), (300, 1243, 90, bf), (8452, 706, 225, f32), (20, 450, 150, f32)):
        for checkpoint in (False, True):
            p = pk.glu_product_plan(0, rows, n_in, Fh, dt, checkpoint)
            tiles = -(-rows // p.tile_rows) * -(-2 * Fh // p.tile_cols)
            assert p.whole + p.cut == tiles and p.tile_cols in (128, 256)
            if checkpoint and p.tile_cols == 128:      # a group lies in two tiles: through the pieces' sum
                assert p.whole == 0
            need = pk.glu_workspace_size(0, rows, n_in, Fh, dt, checkpoint)
            assert need >= (4 * p.cut * p.pieces * p.tile_rows * p.tile_cols if p.pieces > 1 or not p.whole else 0)


def test_binding_refuses(pk):
    x, W = torch.zeros(4, 8), torch.zeros(6, 8)
    d = pk.Drop(0.1, pk.make_key(seed=1, layer=0, step=0, microbatch=0, B=1, S=4, H=8))
    for call in (lambda: pk.glu_forward(x, W), lambda: pk.rms_forward(x), lambda: pk.drop_apply(x, d),
                 lambda: pk.join_forward(x, x), lambda: pk.rms_backward(x, x, torch.zeros(4)),
                 lambda: pk.join_backward(x, None, None, x), lambda: pk.glu_backward_act(x, torch.zeros(4, 16)),
                 lambda: pk.glu_backward_input(x, torch.zeros(8, 3), torch.zeros(4, 6))):
        with pytest.raises(pk.AcscError, match="GPU"):
            call()
    with pytest.raises(pk.AcscError, match="2-D"):
        pk.rms_forward(torch.zeros(3))
    with pytest.raises(pk.AcscError, match="even"):
        pk.glu_forward(x, W[:5])
    with pytest.raises(pk.AcscError, match="dout and dy"):
        pk.join_backward(None, None, x, x)
    with pytest.raises(pk.AcscError, match="make_key"):
        pk._drop_ref(pk.Drop(0.1, None))
    with pytest.raises(pk.AcscError, match="site"):
        pk._drop_ref(pk.Drop(0.1, d.key, -1))
