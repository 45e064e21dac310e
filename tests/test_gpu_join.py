"""Root-mean-square norms, alone and joined with the gate, dropout and residual between two blocks: against 64-bit
references and differences, from tensors and from 8-bit checkpoints."""
import pytest
import torch

from test_gpu_drop import kept, make

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
EPS, SCALE = 1e-5, 0.75
U = 2.0 ** -24
# Of the norm of what a value is the sum of: bf16 outputs take one rounding, at most 2^-8 of each; fp32 sums of H terms
# in a tree of at most 8 CH + 6 + 16 levels (CH <= 8) and a dozen operations on each element.
TOL = {BF16: 2.0 ** -8 + 100 * U, F32: 100 * U}


@pytest.fixture(scope="module")
def pk():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2609_14339_amd as pk
    return pk


def near(got, want, tol, size=None):
    """Within tol of the norm of `size`, the magnitude of the terms that each value is the sum of."""
    got, want = got.double().cpu(), want.double().cpu()
    size = want if size is None else size.double().cpu()
    assert got.shape == want.shape and torch.isfinite(got).all()
    d, n = (got - want).norm(), size.norm()
    assert d <= tol * n + 1e-30, f"{float(d / n):.3e} > {tol:.3e}"


def tensors(rows, H, dtype, pad, seed=0):
    g = torch.Generator().manual_seed(seed + H)
    mat = lambda p: torch.randn(rows, H + p, generator=g).to(dtype).cuda()[:, :H]
    vec = lambda m: (torch.randn(H, generator=g) * 0.2 + m).to(dtype).cuda()
    return dict(r=mat(0), b=mat(pad), dout=mat(pad), dy=mat(0), post=vec(1.0), gate=vec(0.4), pre=vec(1.0))


def ref_forward(t, post, gate, pre, factor):
    r, b = t["r"].double(), t["b"].double()
    out = {}
    if post:
        out["rstd_post"] = 1 / (b.square().mean(1) + EPS).sqrt()
        b = b * out["rstd_post"][:, None] * t["post"].double()
    if gate:
        b = b * t["gate"].double()
    b = b * factor
    out["out"] = SCALE * r + b
    out["size"] = SCALE * r.abs() + b.abs()
    if pre:
        out["rstd_pre"] = 1 / (out["out"].square().mean(1) + EPS).sqrt()
        out["y"] = out["out"] * out["rstd_pre"][:, None] * t["pre"].double()
        out["size_y"] = out["size"] * out["rstd_pre"][:, None] * t["pre"].double().abs()
    return out


def ref_backward(t, x, b, rstd_post, rstd_pre, post, gate, pre, factor, dout=True, scale=SCALE):
    """Gradients, and the magnitude of the terms of each."""
    g = t["dout"].double() if dout else torch.zeros_like(t["dout"]).double()
    size = g.abs()
    out, sizes, rows = {}, {}, g.shape[0]
    if pre:
        rs, dy = rstd_pre.double()[:, None], t["dy"].double()
        h, e = x.double() * rs, dy * t["pre"].double()
        m = (e * h).mean(1, keepdim=True)
        g = g + rs * (e - h * m)
        size = size + rs * (e.abs() + h.abs() * (e * h).abs().mean(1, keepdim=True))
        out["dpre"], sizes["dpre"] = (dy * h).sum(0), (dy * h).abs().sum(0)
    out["dr"], sizes["dr"] = scale * g, scale * size
    u, su = g * factor, size * factor
    h = b.double() * (rstd_post.double()[:, None] if post else 1.0)
    s, ss = (u * h).sum(0), (su * h.abs()).sum(0)
    one = torch.ones_like(t["post"]).double()
    wp, wg = t["post"].double() if post else one, t["gate"].double() if gate else one
    if post:
        out["dpost"], sizes["dpost"] = s * wg, ss * wg.abs()
    if gate:
        out["dgate"], sizes["dgate"] = s * wp, ss * wp.abs()
    e, se = u * wp * wg, su * (wp * wg).abs()
    if post:
        rs = rstd_post.double()[:, None]
        e, se = rs * (e - h * (e * h).mean(1, keepdim=True)), rs * (se + h.abs() * (se * h.abs()).mean(1, keepdim=True))
    out["db"], sizes["db"] = e, se
    return out, sizes


SHAPES = [(1, 1, 0), (1, 64, 0), (2, 7, 0), (5, 500, 3), (129, 512, 0), (7, 1000, 8), (6, 1030, 5), (131, 2048, 0),
          (9, 2049, 0), (33, 4096, 0), (3, 5001, 1), (17, 8192, 0), (2, 8200, 0), (19, 12289, 0), (3, 28672, 0), (2, 32768, 0)]
# (post, gate, pre, p)
FORMS = [(True, True, True, 0.1), (True, False, True, 0.0), (False, True, False, 0.3), (False, False, True, 0.1),
         (True, False, False, 0.0), (False, False, False, 0.5)]


def drop_of(pk, rows, H, p):
    if not p:
        return None, 1.0
    m, up = kept(rows, H, p, 3)
    return make(pk, rows, H, p, 3), (m.double() * float(up)).cuda()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,H,pad", SHAPES)
def test_join_forward(pk, dtype, rows, H, pad):
    t = tensors(rows, H, dtype, pad)
    for post, gate, pre, p in FORMS:
        drop, factor = drop_of(pk, rows, H, p)
        kw = dict(post=t["post"] if post else None, gate=t["gate"] if gate else None, pre=t["pre"] if pre else None,
                  scale=SCALE, drop=drop, eps=EPS)
        j = pk.join_forward(t["r"], t["b"], **kw, checkpoint=True)
        ref = ref_forward(t, post, gate, pre, factor)
        near(j.out, ref["out"], TOL[dtype], ref["size"])
        if post:
            near(j.rstd_post, ref["rstd_post"], TOL[F32])
        if pre:
            # near 0 for a row whose terms cancel: compared at the size of the terms
            near(j.y, ref["y"], TOL[dtype], ref["size_y"])
        assert (j.rstd_post is None) == (not post) and (j.rstd_pre is None) == (j.y is None) == (not pre)
        want = pk.q8_encode(t["b"])
        assert torch.equal(j.q_b.codes, want.codes) and torch.equal(j.q_b.scales, want.scales)
        if dtype == F32:
            want = pk.q8_encode(j.out)
            assert torch.equal(j.q_out.codes, want.codes) and torch.equal(j.q_out.scales, want.scales)
        else:                      # coded before the rounding to bf16
            v, top = pk.q8_decode(j.q_out, F32).double(), j.q_out.scales.repeat_interleave(128, 1)[:, :H].double()
            assert ((v - ref["out"]).abs() <= 0.51 * top + 100 * U * ref["size"]).all()
        for part in ("out", "b"):
            k = pk.join_forward(t["r"], t["b"], **kw, checkpoint=part)
            assert (k.q_out is None) == (part == "b") and (k.q_b is None) == (part == "out")
            q, want = (k.q_out, j.q_out) if part == "out" else (k.q_b, j.q_b)
            assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales) and torch.equal(k.out, j.out)
        k = pk.join_forward(t["r"], t["b"], **kw)
        assert torch.equal(k.out, j.out) and (k.y is None or torch.equal(k.y, j.y)) and k.q_out is k.q_b is None


@pytest.mark.parametrize("kept_as", ["whole", "q8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,H,pad", SHAPES + [(3000, 256, 0), (1300, 4100, 4), (700, 8192, 0), (600, 12000, 0), (530, 17000, 0)])
def test_join_backward(pk, dtype, rows, H, pad, kept_as):
    t = tensors(rows, H, dtype, pad)
    for post, gate, pre, p in FORMS[:2] if rows >= 500 else FORMS:
        drop, factor = drop_of(pk, rows, H, p)
        j = pk.join_forward(t["r"], t["b"], t["post"] if post else None, t["gate"] if gate else None, t["pre"] if pre else None,
                            SCALE, drop, EPS, checkpoint=True)
        x, b, vx, vb = (j.out, t["b"], j.out, t["b"]) if kept_as == "whole" else \
            (j.q_out, j.q_b, pk.q8_decode(j.q_out, F32), pk.q8_decode(j.q_b, F32))
        args = (t["dout"], t["dy"] if pre else None, x if pre else None, b if post or gate else None, j.rstd_post, j.rstd_pre,
                t["post"] if post else None, t["gate"] if gate else None, t["pre"] if pre else None, SCALE, drop)
        d = pk.join_backward(*args)
        want, size = ref_backward(t, vx, vb, j.rstd_post, j.rstd_pre, post, gate, pre, factor)
        near(d.dr, want["dr"], TOL[dtype], size["dr"])
        near(d.db, want["db"], TOL[dtype], size["db"])
        for name in ("dpost", "dgate", "dpre"):
            got = getattr(d, name)
            assert (got is None) == (name not in want)
            if got is not None:    # at most `rows` additions, and the roundings of each term on its way
                assert ((got.double() - want[name]).abs() <= U * (rows + 200) * size[name] + 1e-30).all(), name
        again = pk.join_backward(*args)
        assert all(u is v or torch.equal(u, v) for u, v in zip(again, d))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,H,pad", SHAPES)
def test_rms_norm(pk, dtype, rows, H, pad):
    t = tensors(rows, H, dtype, pad)
    x, gamma, dy, add = t["b"], t["pre"], t["dy"], t["dout"]
    y, rstd, q = pk.rms_forward(x, gamma, EPS, checkpoint=True)
    rs = 1 / (x.double().square().mean(1) + EPS).sqrt()
    near(rstd, rs, TOL[F32])
    near(y, x.double() * rs[:, None] * gamma.double(), TOL[dtype])
    want = pk.q8_encode(x)
    assert torch.equal(q.codes, want.codes) and torch.equal(q.scales, want.scales)
    assert torch.equal(pk.rms_forward(x, gamma, EPS)[0], y)
    assert torch.equal(pk.rms_recompute(x, rstd, gamma, dtype), y)
    v = pk.q8_decode(q, F32)
    near(pk.rms_recompute(q, rstd, gamma, dtype), v.double() * rstd.double()[:, None] * gamma.double(), TOL[dtype])
    near(pk.rms_forward(x, None, EPS)[0], x.double() * rs[:, None], TOL[dtype])
    for src, value in ((x, x), (q, v)):
        dx, dg = pk.rms_backward(dy, src, rstd, gamma, add=add)
        ref, size = ref_backward(dict(t, dout=add), value, value, None, rstd, False, False, True, 1.0, scale=1.0)
        near(dx, ref["dr"], TOL[dtype], size["dr"])
        assert ((dg.double() - ref["dpre"]).abs() <= U * (rows + 100) * size["dpre"] + 1e-30).all()
        dx2, none = pk.rms_backward(dy, src, rstd, gamma, add=add, weights=False)
        assert none is None and torch.equal(dx2, dx)


def test_gradients_without_one_of_the_two_incoming(pk):
    rows, H = 37, 1500
    t = tensors(rows, H, F32, 0)
    drop, factor = drop_of(pk, rows, H, 0.2)
    j = pk.join_forward(t["r"], t["b"], t["post"], t["gate"], t["pre"], SCALE, drop, EPS)
    args = (j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE, drop)
    d = pk.join_backward(None, t["dy"], *args)
    want, size = ref_backward(t, j.out, t["b"], j.rstd_post, j.rstd_pre, True, True, True, factor, dout=False)
    near(d.dr, want["dr"], TOL[F32], size["dr"])
    near(d.db, want["db"], TOL[F32], size["db"])
    d = pk.join_backward(t["dout"], None, None, *args[1:])
    want, size = ref_backward(t, None, t["b"], j.rstd_post, None, True, True, False, factor)
    near(d.db, want["db"], TOL[F32], size["db"])
    assert d.dpre is None and d.dpost is not None


def test_in_place_accumulating_and_strided(pk):
    rows, H = 300, 1000
    t = tensors(rows, H, BF16, 0)
    drop, _ = drop_of(pk, rows, H, 0.1)
    kw = dict(post=t["post"], gate=t["gate"], pre=t["pre"], scale=SCALE, drop=drop, eps=EPS)
    j = pk.join_forward(t["r"], t["b"], **kw)
    r, b = t["r"].clone(), t["b"].clone()
    k = pk.join_forward(r, b, **kw, out=r, y=b)
    assert torch.equal(r, j.out) and torch.equal(b, j.y) and k.out is r and k.y is b
    wide = torch.full((rows, H + 9), 5.0, dtype=BF16, device="cuda")
    pk.join_forward(t["r"], t["b"], **kw, out=wide[:, :H])
    assert torch.equal(wide[:, :H], j.out) and (wide[:, H:] == 5).all()
    args = (j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE, drop)
    d = pk.join_backward(t["dout"], t["dy"], *args)
    g, dy = t["dout"].clone(), t["dy"].clone()
    base = [torch.randn(H, device="cuda") for _ in range(3)]
    sums = [s.clone() for s in base]
    pk.join_backward(g, dy, *args, dr=g, db=dy, dpost=sums[0], dgate=sums[1], dpre=sums[2], accumulate=True)
    assert torch.equal(g, d.dr) and torch.equal(dy, d.db)
    assert all(torch.equal(s, o + e) for s, o, e in zip(sums, base, (d.dpost, d.dgate, d.dpre)))


def test_masked_and_non_finite_rows(pk):
    """A row that the mask left empty, an empty branch, and a row that is not finite, which stays alone."""
    rows, H = 40, 1500
    t = tensors(rows, H, F32, 0)
    t["r"][3] = 0
    t["b"][3] = 0
    t["b"][4] = 0
    drop, factor = drop_of(pk, rows, H, 0.1)
    kw = dict(post=t["post"], gate=t["gate"], pre=t["pre"], scale=SCALE, drop=drop, eps=EPS)
    j = pk.join_forward(t["r"], t["b"], **kw)
    assert (j.out[3] == 0).all() and (j.y[3] == 0).all() and torch.equal(j.out[4], SCALE * t["r"][4])
    args = (j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE, drop)
    d = pk.join_backward(t["dout"], t["dy"], j.out, t["b"], *args)
    assert all(torch.isfinite(v).all() for v in d)
    bad = dict(t, b=t["b"].clone(), r=t["r"].clone())
    bad["b"][13, 700], bad["r"][20, 2] = float("nan"), float("inf")
    k = pk.join_forward(bad["r"], bad["b"], **kw)
    ok = [i for i in range(rows) if i not in (13, 20)]
    assert torch.equal(k.out[ok], j.out[ok]) and torch.equal(k.y[ok], j.y[ok])
    assert torch.isnan(k.y[13]).all() and not torch.isfinite(k.y[20]).all()
    e = pk.join_backward(t["dout"], t["dy"], k.out, bad["b"], k.rstd_post, k.rstd_pre, *args[2:])
    assert torch.equal(e.dr[ok], d.dr[ok]) and torch.equal(e.db[ok], d.db[ok])


def test_no_rows(pk):
    e, g = torch.empty(0, 96, device="cuda"), torch.ones(96, device="cuda")
    drop = pk.Drop(0.1, pk.make_key(seed=1, layer=0, step=0, microbatch=0, B=4, S=0, H=96))
    j = pk.join_forward(e, e, g, g, g, 1.0, drop, EPS, checkpoint=True)
    assert j.out.shape == j.y.shape == (0, 96) and j.rstd_post.shape == (0,)
    d = pk.join_backward(e, e, e, e, j.rstd_post, j.rstd_pre, g, g, g, 1.0, drop)
    assert d.dr.shape == (0, 96) and all((v == 0).all() for v in (d.dpost, d.dgate, d.dpre))
    y, rstd, q = pk.rms_forward(e, g, EPS, checkpoint=True)
    dx, dg = pk.rms_backward(e, q, rstd, g)
    assert y.shape == dx.shape == (0, 96) and (dg == 0).all()


@pytest.mark.parametrize("H", [96, 3000])
def test_gradients_against_differences(pk, H):
    """Central differences of the fp32 forward pass along random directions: truncation h^2 / 6 of a third derivative
    of order 1, rounding 2^-24 |f| / h per output; h = 2^-7 leaves both under 1e-4 of the sums compared."""
    rows = 8
    t = tensors(rows, H, F32, 0)
    drop, _ = drop_of(pk, rows, H, 0.2)
    names = ("r", "b", "post", "gate", "pre")

    def f(v):
        j = pk.join_forward(*v[:4], pre=v[4], scale=SCALE, drop=drop, eps=EPS)
        return (j.out.double() * t["dout"].double()).sum() + (j.y.double() * t["dy"].double()).sum()
    v = [t[n] for n in names]
    j = pk.join_forward(*v[:4], pre=v[4], scale=SCALE, drop=drop, eps=EPS)
    d = pk.join_backward(t["dout"], t["dy"], j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE, drop)
    h = 2.0 ** -7
    for i, grad in enumerate((d.dr, d.db, d.dpost, d.dgate, d.dpre)):
        u = torch.randn(grad.shape, generator=torch.Generator().manual_seed(i)).cuda()
        at = lambda s: [w + s * h * u if k == i else w for k, w in enumerate(v)]
        diff = (f(at(1)) - f(at(-1))) / (2 * h)
        scale = float((grad.double() * u.double()).norm())
        assert abs(float(diff - (grad.double() * u.double()).sum())) <= 2e-3 * scale, names[i]


def test_streams_and_graphs(pk):
    rows, H = 512, 1024
    t = tensors(rows, H, BF16, 0)
    drop, _ = drop_of(pk, rows, H, 0.1)
    kw = dict(post=t["post"], gate=t["gate"], pre=t["pre"], scale=SCALE, drop=drop, eps=EPS)

    def both(s=None):
        j = pk.join_forward(t["r"], t["b"], **kw, stream=s)
        return [*j[:4], *pk.join_backward(t["dout"], t["dy"], j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"],
                                          t["pre"], SCALE, drop, stream=s)]
    want = both()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = both(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for i in range(3):
        t["b"].copy_(torch.randn(rows, H, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, both()))


@pytest.mark.parametrize("kept_as", ["whole", "q8"])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("H", [700, 3000, 8192, 9001, 17000])
def test_gradients_in_the_place_of_every_input(pk, dtype, H, kept_as):
    """dr and db may each take the place of any tensor that the call reads."""
    rows = 600
    t = tensors(rows, H, dtype, 0)
    drop = make(pk, rows, H, 0.1, 3)
    j = pk.join_forward(t["r"], t["b"], t["post"], t["gate"], t["pre"], SCALE, drop, EPS, checkpoint=True)
    src = dict(dout=t["dout"], dy=t["dy"], out=j.out, b=t["b"])

    def call(v, **places):
        out, b = (v["out"], v["b"]) if kept_as == "whole" else (j.q_out, j.q_b)
        return pk.join_backward(v["dout"], v["dy"], out, b, j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE, drop,
                                **places)
    want = call(src)
    names = ["dout", "dy", "out", "b"] if kept_as == "whole" else ["dout", "dy"]
    for i, name in enumerate(names):
        v = {k: s.clone() for k, s in src.items()}
        d = call(v, dr=v[name], db=v[names[i - 1]])
        assert all(torch.equal(a, b) for a, b in zip(d, want)), name


def test_a_stream_that_wants_no_gradient(pk):
    """dr == NULL: the other gradients, and nothing is written in its place."""
    for H in (300, 9001):
        rows = 50
        t = tensors(rows, H, F32, 0)
        j = pk.join_forward(t["r"], t["b"], t["post"], t["gate"], t["pre"], SCALE, None, EPS)
        want = pk.join_backward(t["dout"], t["dy"], j.out, t["b"], j.rstd_post, j.rstd_pre, t["post"], t["gate"], t["pre"], SCALE)
        db, sums = torch.empty_like(want.db), [torch.empty(H, device="cuda") for _ in range(3)]
        ws = torch.empty(pk.join_workspace_size(rows, H), dtype=torch.uint8, device="cuda")
        p = lambda v: v.data_ptr()
        rc = pk.lib.join_backward(p(t["dout"]), t["dout"].stride(0), p(t["dy"]), H, p(j.out), H, None, p(t["b"]), t["b"].stride(0),
                                  None, pk.F32, rows, H, p(t["post"]), p(t["gate"]), SCALE, None, p(t["pre"]), p(j.rstd_post),
                                  p(j.rstd_pre), None, 0, p(db), H, *map(p, sums), 0, p(ws), ws.numel(), pk._raw_stream())
        assert rc == 0, pk.lib.acsc_last_error()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((db, *sums), want[1:]))
