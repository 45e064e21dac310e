"""The operators of a pipeline stage's feed-forward block, as timed cases: layer norm, the matrix product with bias,
activation and residual in its epilogue, and activation checkpoints in 8 bits, each with its gradients.

Between two masked boundaries a stage runs x + W2 act(W1 norm(x) + b1) + b2 on its tokens and keeps, for every
microbatch in flight, what the backward pass reads: the block's input and the pre-activation, both as 8-bit
checkpoints (one scale per 128 columns of a row).  Each case is one pass through one of these operators.

Where `own` is false, `run` computes them from elementary torch operations in 32 bits, rounded once at the end;
where it is true, through the library's entry points.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 128
EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # the norm of a toy stage (2 x 64 tokens): launch latency
        dict(name="norm-tiny", kind="norm", dtype="f32", rows=128, H=256, ckpt=False, pad=0),
        # the norm at the start of a 70B-class block, writing the block's checkpoint in the same pass
        dict(name="norm-ckpt-70b", kind="norm", dtype="bf16", rows=16384, H=8192, ckpt=True, pad=0),
        # the norm's backward pass in a 1B-class block that keeps its input whole, with the residual branch's gradient
        dict(name="norm-bwd-1b", kind="norm-bwd", dtype="bf16", rows=16384, H=2048, ckpt=False, pad=0),
        # the same in an 8B-class block that keeps its input in 8 bits
        dict(name="norm-bwd-ckpt-8b", kind="norm-bwd", dtype="bf16", rows=16384, H=4096, ckpt=True, pad=0),
        # one token through an 8B-class up projection (evaluation): the weights' bytes
        dict(name="linear-token-8b", kind="linear", dtype="bf16", rows=1, n_in=4096, n_out=14336, act="gelu",
             res=False, ckpt=False, pad=0),
        # the up projection of a 1B-class block (8 x 2048 tokens), keeping its pre-activation in 8 bits
        dict(name="linear-up-1b", kind="linear", dtype="bf16", rows=16384, n_in=2048, n_out=8192, act="gelu",
             res=False, ckpt=True, pad=0),
        # the down projection of a 70B-class block with the residual added
        dict(name="linear-down-70b", kind="linear", dtype="bf16", rows=8192, n_in=28672, n_out=8192, act="none",
             res=True, ckpt=False, pad=0),
        # an fp32 product of odd sizes with every part of the epilogue, its input a slice of a wider tensor
        dict(name="linear-odd-f32", kind="linear", dtype="f32", rows=1237, n_in=1000, n_out=4099, act="silu",
             res=True, ckpt=False, pad=5),
        # the down projection's backward pass in an 8B-class block (2 x 4096 tokens): the gradient through the kept
        # pre-activation, and the weights' gradient
        dict(name="linear-bwd-8b", kind="linear-bwd", dtype="bf16", rows=8192, n_in=14336, n_out=4096, act="gelu",
             ckpt=True, pad=0),
        # the same with a ragged batch, widths that fill no tile, and whole activations
        dict(name="linear-bwd-odd", kind="linear-bwd", dtype="bf16", rows=999, n_in=3001, n_out=1100, act="silu",
             ckpt=False, pad=0),
        # an 8-bit checkpoint of a 70B-class hidden activation, written and read back through its activation function
        dict(name="ckpt-70b", kind="ckpt", dtype="bf16", rows=8192, H=28672, act="gelu", pad=0),
        # a small ragged one
        dict(name="ckpt-odd", kind="ckpt", dtype="bf16", rows=771, H=1023, act="none", pad=2),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths are multiples of 64 more often than not, as models' are."""
    n = _log(rng, lo, hi)
    return max(lo, n // 64 * 64) if rng.random() < 0.6 else n


def draw(rng):
    kind = rng.choice(["norm", "norm-bwd", "linear", "linear", "linear-bwd", "linear-bwd", "ckpt"])
    case = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), pad=rng.choice([0, 0, 0, 8, 5]))
    if kind in ("norm", "norm-bwd", "ckpt"):
        H = _width(rng, 64, 28672)
        case.update(rows=min(_log(rng, 1, 32768), (1 << 27) // H), H=H)
    else:
        n_in, n_out = _width(rng, 64, 16384), _width(rng, 64, 16384)
        most = (1 << 39) * 3 // 2 // (n_in * n_out)
        case.update(rows=max(1, min(_log(rng, 1, 16384), most)), n_in=n_in, n_out=n_out,
                    act=rng.choice(["none", "relu", "gelu", "silu"]))
    if kind == "linear":
        case["res"] = rng.random() < 0.5
    if kind == "ckpt":
        case["act"] = rng.choice(["none", "gelu", "silu"])
    else:
        # a product's fp32 sums depend on their order, and a code at a tie with them: no fp32 outputs through codes
        case["ckpt"] = rng.random() < 0.5 and (case["dtype"] == "bf16" or kind == "norm-bwd")
    return case


def _gen(seed, *ids):
    for v in ids:
        seed = (seed * 1000003 + v + 1) % (1 << 62)
    return torch.Generator(device="cuda").manual_seed(seed)


def _slice(t, pad):
    """t as the first columns of a wider tensor."""
    if not pad:
        return t
    wide = torch.zeros(t.shape[0], t.shape[1] + pad, dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _hidden(rows, H, dt, pad, g):
    """Hidden states: unit scale, offsets that differ by column, and a few columns that are 20 times as large."""
    scale = torch.ones(H, device="cuda")
    scale[torch.randperm(H, generator=g, device="cuda")[:max(1, H // 256)]] = 20.0
    x = torch.randn(rows, H, generator=g, device="cuda")
    x.add_(torch.randn(H, generator=g, device="cuda").mul_(0.3).add_(0.5)).mul_(scale)
    return _slice(x.to(dt), pad)


def _normal(rows, H, dt, pad, g, scale=1.0):
    return _slice(torch.randn(rows, H, generator=g, device="cuda").mul_(scale).to(dt), pad)


def _codes(x):
    """An 8-bit checkpoint of x: codes, and one scale for each 128 columns of a row."""
    rows, H = x.shape
    n = -(-H // GROUP)
    v = torch.zeros(rows, n * GROUP, device=x.device)
    v[:, :H] = x
    v = v.view(rows, n, GROUP)
    top = v.abs().amax(2, keepdim=True)
    most = torch.full_like(top, 127.0)         # quotients of tensors: those with a plain number go by its reciprocal
    codes = torch.round(v * torch.where(top > 0, most / top, 0.0)).clamp(-127, 127)
    return codes.view(rows, n * GROUP)[:, :H].to(torch.int8).contiguous(), (top / most).view(rows, n)


def _values(codes, scales):
    return codes.to(scales.dtype) * scales.repeat_interleave(GROUP, 1)[:, :codes.shape[1]]


def prepare(case, seed):
    kind, dt, pad, rows = case["kind"], DTYPES[case["dtype"]], case["pad"], case["rows"]
    g = _gen(seed, 1)
    st = dict(case=case)
    if kind in ("norm", "norm-bwd"):
        H = case["H"]
        st["x"] = _hidden(rows, H, dt, pad, g)
        st["gamma"] = torch.randn(H, generator=g, device="cuda").mul_(0.1).add_(1.0).to(dt)
        if kind == "norm":
            st["beta"] = torch.randn(H, generator=g, device="cuda").mul_(0.1).to(dt)
        else:
            x = st["x"].float()
            st["mean"] = x.mean(1)
            st["rstd"] = torch.rsqrt((x - st["mean"][:, None]).square().mean(1) + EPS)
            st["dy"] = _normal(rows, H, dt, 0, g)
            st["add"] = _normal(rows, H, dt, 0, g)
            if case["ckpt"]:
                st["codes"], st["scales"] = _codes(st.pop("x"))
    elif kind == "ckpt":
        st["x"] = _hidden(rows, case["H"], dt, pad, g)
    else:
        n_in, n_out = case["n_in"], case["n_out"]
        st["W"] = _normal(n_out, n_in, dt, 0, g, 1 / math.sqrt(n_in))
        if kind == "linear":
            st["x"] = _normal(rows, n_in, dt, pad, g)
            st["b"] = _normal(1, n_out, dt, 0, g, 0.1)[0]
            st["res"] = _normal(rows, n_out, dt, 0, g) if case["res"] else None
        else:
            st["dz"] = _normal(rows, n_out, dt, pad, g)
            st["z"] = _normal(rows, n_in, dt, 0, g)
            if case["ckpt"]:
                st["codes"], st["scales"] = _codes(st.pop("z"))
    return st


def _act(z, act):
    if act == "relu":
        return torch.relu(z)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_grad(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2 * math.pi))
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return None


def _run_own(st):
    import paper_2609_14339_amd as acsc

    case, kind = st["case"], st["case"]["kind"]
    dt = DTYPES[case["dtype"]]
    if kind == "norm":
        y, mean, rstd, q = acsc.ln_forward(st["x"], st["gamma"], st["beta"], EPS, checkpoint=case["ckpt"])
        out = dict(y=y, mean=mean, rstd=rstd)
        if case["ckpt"]:
            out["kept"] = acsc.q8_decode(q, dt)
        return out
    if kind == "norm-bwd":
        src = acsc.Q8(st["codes"], st["scales"]) if case["ckpt"] else st["x"]
        dx, dgamma, dbeta = acsc.ln_backward(st["dy"], src, st["mean"], st["rstd"], st["gamma"], add=st["add"])
        return dict(dx=dx, dgamma=dgamma, dbeta=dbeta)
    if kind == "ckpt":
        return acsc.q8_decode(acsc.q8_encode(st["x"]), dt, act=case["act"])
    if kind == "linear":
        y, q = acsc.lin_forward(st["x"], st["W"], st["b"], act=case["act"], residual=st["res"],
                                keep="q8" if case["ckpt"] else None)
        return dict(y=y, kept=acsc.q8_decode(q, dt)) if case["ckpt"] else dict(y=y)
    z = acsc.Q8(st["codes"], st["scales"]) if case["ckpt"] else st["z"]
    dx = acsc.lin_backward_input(st["dz"], st["W"], act=case["act"], z=z)
    dW, db = acsc.lin_backward_weight(st["dz"], z, act=case["act"], dw_dtype=dt)
    return dict(dx=dx, dW=dW, db=db)


def run(st):
    if own:
        return _run_own(st)
    case, kind = st["case"], st["case"]["kind"]
    dt = DTYPES[case["dtype"]]
    if kind == "norm":
        x = st["x"].float()
        mean = x.mean(1)
        c = x - mean[:, None]
        rstd = torch.rsqrt(c.square().mean(1) + EPS)
        out = dict(y=(c * rstd[:, None] * st["gamma"].float() + st["beta"].float()).to(dt), mean=mean, rstd=rstd)
        if case["ckpt"]:
            out["kept"] = _values(*_codes(x)).to(dt)
        return out
    if kind == "norm-bwd":
        x = _values(st["codes"], st["scales"]) if case["ckpt"] else st["x"].float()
        dy = st["dy"].float()
        h = (x - st["mean"][:, None]) * st["rstd"][:, None]
        g = dy * st["gamma"].float()
        dx = st["rstd"][:, None] * (g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True))
        return dict(dx=(dx + st["add"].float()).to(dt), dgamma=(dy * h).sum(0), dbeta=dy.sum(0))
    if kind == "ckpt":
        return _act(_values(*_codes(st["x"].float())), case["act"]).to(dt)
    if kind == "linear":
        z = torch.mm(st["x"].float(), st["W"].float().t()) + st["b"].float()
        y = _act(z, case["act"])
        if case["res"]:
            y = y + st["res"].float()
        return dict(y=y.to(dt), kept=_values(*_codes(z)).to(dt)) if case["ckpt"] else dict(y=y.to(dt))
    z = _values(st["codes"], st["scales"]) if case["ckpt"] else st["z"].float()
    dz = st["dz"].float()
    dx = torch.mm(dz, st["W"].float())
    if case["act"] != "none":
        dx = dx * _act_grad(z, case["act"])
    dW = torch.mm(dz.t(), _act(z, case["act"]))
    return dict(dx=dx.to(dt), dW=dW.to(dt), db=dz.sum(0))


def work(case):
    """Bytes that each pass reads and writes once, and the products' operations."""
    kind, e, rows = case["kind"], 2 if case["dtype"] == "bf16" else 4, case["rows"]
    q = 1 + 4 / GROUP
    if kind in ("norm", "norm-bwd", "ckpt"):
        n = rows * case["H"]
        if kind == "norm":
            return dict(bytes=n * (2 * e + (q + e if case["ckpt"] else 0)) + 2 * e * case["H"] + 8 * rows, flops=8 * n)
        if kind == "ckpt":
            return dict(bytes=n * (2 * e), flops=4 * n)
        return dict(bytes=n * (3 * e + (q if case["ckpt"] else e)) + (e + 8) * case["H"] + 8 * rows, flops=14 * n)
    n_in, n_out = case["n_in"], case["n_out"]
    if kind == "linear":
        outs = rows * n_out * (e + (e if case["res"] else 0) + (e if case["ckpt"] else 0))
        return dict(bytes=e * (rows * n_in + n_in * n_out + n_out) + outs, flops=2 * rows * n_in * n_out)
    kept = q if case["ckpt"] else e
    return dict(bytes=e * (rows * n_out + 2 * n_in * n_out + rows * n_in) + kept * rows * n_in + 4 * n_out,
                flops=4 * rows * n_in * n_out)


def _codes64(x):
    """The checkpoint's values from its definition, in 64 bits."""
    rows, H = x.shape
    full = torch.nn.functional.pad(x.double(), (0, -H % GROUP)).reshape(rows, -1, GROUP)
    step = full.abs().max(dim=2, keepdim=True).values / 127
    whole = torch.where(step > 0, full / step, torch.zeros_like(full)).round().clamp(-127, 127)
    return (whole * step).reshape(rows, -1)[:, :H]


def _pair64(z, act):
    """(act(z), act'(z)) in 64 bits."""
    if act == "none":
        return z, torch.ones_like(z)
    if act == "relu":
        on = (z > 0).double()
        return z * on, on
    if act == "silu":
        s = torch.sigmoid(z)
        return z * s, s + z * s * (1 - s)
    phi = 0.5 * torch.erfc(-z / math.sqrt(2))
    return z * phi, phi + z * torch.exp(-z.square() / 2) / math.sqrt(2 * math.pi)


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "ckpt":
        return _pair64(_codes64(st["x"]), case["act"])[0]
    if kind == "norm":
        x = st["x"].double()
        var, mean = torch.var_mean(x, 1, correction=0)
        rstd = 1 / torch.sqrt(var + EPS)
        y = torch.addcmul(st["beta"].double(), (x - mean[:, None]).mul_(rstd[:, None]), st["gamma"].double())
        out = dict(y=y, mean=mean, rstd=rstd)
        if case["ckpt"]:
            out["kept"] = _codes64(x)
        return out
    if case.get("ckpt") and kind != "linear":
        src = st["codes"].double() * st["scales"].double().repeat_interleave(GROUP, 1)[:, :st["codes"].shape[1]]
    else:
        src = st["z" if kind == "linear-bwd" else "x"].double()
    if kind == "norm-bwd":
        # dx = r (I - 1 1'/H - h h'/H) (dy gamma), row by row
        r, H, dy = st["rstd"].double()[:, None], case["H"], st["dy"].double()
        h = src.sub_(st["mean"].double()[:, None]).mul_(r)
        u = dy * st["gamma"].double()
        dx = r * (u - (u.sum(1, keepdim=True) + h * (u * h).sum(1, keepdim=True)) / H) + st["add"].double()
        return dict(dx=dx, dgamma=torch.einsum("ij,ij->j", dy, h), dbeta=dy.sum(0))
    if kind == "linear":
        z = torch.addmm(st["b"].double(), src, st["W"].double().t())
        y = _pair64(z, case["act"])[0]
        if case["res"]:
            y = y + st["res"].double()
        return dict(y=y, kept=_codes64(z)) if case["ckpt"] else dict(y=y)
    a, slope = _pair64(src, case["act"])
    dz = st["dz"].double()
    return dict(dx=(dz @ st["W"].double()).mul_(slope), dW=dz.t() @ a, db=dz.sum(0))
