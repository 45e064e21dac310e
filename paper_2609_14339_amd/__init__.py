"""Python binding of libacsc.so (include/acsc.h): argument marshalling only.

Every step of the hot path runs in the HIP library; this module turns torch
tensors into device pointers and the current HIP stream, calls the C entry
point of the same name, and raises ``AcscError`` on a non-zero return code.
There is no fallback: if the library is not built, importing this package
raises ``ImportError``.

``stream=`` runs a call on a stream other than the current one.  The caller
orders that stream after what produced the inputs, and whoever reads the
outputs after that stream; the memory that a call allocates, and that of the
tensors in its arguments, is taken care of here.  (A batched call's items, with
their outputs and workspaces, stay the caller's to keep.)
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import NamedTuple, Optional, Union

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libacsc.so")

F32, BF16 = 0, 1
SC_KMAX = 192

ACSC_OK, ACSC_EINVAL, ACSC_EDTYPE, ACSC_EALIGN, ACSC_EHIP, ACSC_ENOSPC, ACSC_ENOCONV = 0, -1, -2, -3, -4, -5, -6


class AcscError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"acsc error {code}: {msg}")
        self.code = code


class MaskKey(C.Structure):
    """ac_mask_key: the fields of the paper's g(layer, step, B, S, H) plus a
    seed and a microbatch id."""
    _fields_ = [("seed", C.c_uint64), ("step", C.c_uint64), ("layer", C.c_uint32),
                ("microbatch", C.c_uint32), ("B", C.c_uint32), ("S", C.c_uint32),
                ("H", C.c_uint32)]


class ScMatrix(C.Structure):
    """sc_matrix: one weight matrix of a batched sc_* call."""
    _fields_ = [("G", C.c_void_p), ("M", C.c_void_p), ("m", C.c_int), ("n", C.c_int),
                ("U", C.c_void_p), ("s", C.c_void_p), ("V", C.c_void_p), ("d", C.c_void_p),
                ("V_warm", C.c_void_p), ("G_proj", C.c_void_p), ("ws", C.c_void_p),
                ("ws_bytes", C.c_size_t)]


class AdamwState(C.Structure):
    """sc_adamw_state: one matrix's fp32 weights and Adam moments (in place)."""
    _fields_ = [("W", C.c_void_p), ("m1", C.c_void_p), ("m2", C.c_void_p)]


class AdamwHparams(C.Structure):
    """sc_adamw_hparams: one step's AdamW hyperparameters."""
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("step", C.c_int64), ("max_norm", C.c_float)]


class PsgdMatrix(C.Structure):
    """psgd_matrix: one matrix of a PowerSGD call."""
    _fields_ = [("G", C.c_void_p), ("E", C.c_void_p), ("P", C.c_void_p), ("Q", C.c_void_p),
                ("out", C.c_void_p), ("m", C.c_int), ("n", C.c_int), ("ws", C.c_void_p),
                ("ws_bytes", C.c_size_t)]


class _Q8Tensor(C.Structure):
    """q8_tensor: the device arrays of an 8-bit checkpoint."""
    _fields_ = [("codes", C.c_void_p), ("scales", C.c_void_p), ("ld_codes", C.c_int64), ("ld_scales", C.c_int64)]


class _LinPlan(C.Structure):
    """lin_plan: how a product of a linear layer is cut."""
    _fields_ = [("tile_rows", C.c_int), ("tile_cols", C.c_int), ("whole", C.c_int64), ("cut", C.c_int64), ("pieces", C.c_int)]


class LinPlan(NamedTuple):
    """A product in tiles of tile_rows x tile_cols, `whole` of them in one
    piece and `cut` of them in `pieces`; 0 x 0: a product for few rows."""
    tile_rows: int
    tile_cols: int
    whole: int
    cut: int
    pieces: int


class Q8(NamedTuple):
    """An 8-bit checkpoint of a [rows, H] tensor: codes int8 [rows, H] and one
    fp32 scale for each 128 columns of a row, scales [rows, ceil(H / 128)]."""
    codes: torch.Tensor
    scales: torch.Tensor


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                          "(or python paper_2609_14339_amd/build.py)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, u64, f32, sz = C.c_void_p, C.c_int, C.c_int64, C.c_uint64, C.c_float, C.c_size_t
    lib.acsc_last_error.restype = C.c_char_p
    lib.acsc_last_error.argtypes = []
    lib.acsc_version.restype = i32
    lib.ac_keep_count.restype = i32
    lib.ac_keep_count.argtypes = [i32, C.c_double, C.POINTER(i32)]
    lib.ac_mask_pack.restype = i32
    lib.ac_mask_pack.argtypes = [vp, i32, i64, i32, i64, i32, C.POINTER(MaskKey), vp, vp, vp]
    lib.ac_unpack_scatter.restype = i32
    lib.ac_unpack_scatter.argtypes = [vp, vp, i32, i64, i32, i32, C.POINTER(MaskKey), f32, vp,
                                      i64, vp]
    lib.ac_mask_pack_batched.restype = i32
    lib.ac_mask_pack_batched.argtypes = [vp, i32, i32, i64, i32, i64, i64, i32, C.POINTER(MaskKey), vp, i64,
                                         vp, vp, i64, vp]
    lib.ac_unpack_scatter_batched.restype = i32
    lib.ac_unpack_scatter_batched.argtypes = [vp, i64, i32, i32, i64, i32, i32, C.POINTER(MaskKey), vp, vp, i64,
                                              f32, vp, i64, i64, vp]
    lib.ac_bern_mask.restype = i32
    lib.ac_bern_mask.argtypes = [i64, i32, C.c_double, C.POINTER(MaskKey), vp, vp, vp]
    lib.ac_bern_pack.restype = i32
    lib.ac_bern_pack.argtypes = [vp, i32, i64, i32, i64, vp, vp, vp, vp, i64, vp]
    lib.ac_bern_unpack.restype = i32
    lib.ac_bern_unpack.argtypes = [vp, i32, i64, i32, vp, vp, i64, f32, vp, i64, vp]
    lib.sc_workspace_size.restype = i32
    lib.sc_workspace_size.argtypes = [i32, i32, i32, i32, i32, C.POINTER(sz)]
    lib.sc_build_prior.restype = i32
    lib.sc_build_prior.argtypes = [vp, i32, vp, i32, i32, f32, i32, i32, i32, f32, vp, u64,
                                   vp, vp, vp, vp, vp, sz, vp]
    lib.sc_correct.restype = i32
    lib.sc_correct.argtypes = [vp, i32, i32, i32, vp, vp, vp, i32, f32, vp, vp, sz, vp]
    lib.sc_correct_static.restype = i32
    lib.sc_correct_static.argtypes = [vp, i32, i32, i32, vp, vp, vp, i32, f32, vp, vp]
    for fn in (lib.sc_build_prior_batched, lib.sc_build_subspace_batched, lib.sc_build_ritz_batched):
        fn.restype = i32
        fn.argtypes = [i32, C.POINTER(ScMatrix), i32, f32, i32, i32, i32, f32, u64, vp]
    lib.sc_build_status.restype = i32
    lib.sc_build_status.argtypes = [i32, C.POINTER(ScMatrix), vp, vp, vp]
    lib.sc_correct_batched.restype = i32
    lib.sc_correct_batched.argtypes = [i32, C.POINTER(ScMatrix), i32, i32, f32, vp]
    lib.sc_adamw_workspace_size.restype = i32
    lib.sc_adamw_workspace_size.argtypes = [i32, i32, i32, i32, C.POINTER(sz)]
    lib.sc_correct_adamw_batched.restype = i32
    lib.sc_correct_adamw_batched.argtypes = [i32, C.POINTER(ScMatrix), C.POINTER(AdamwState), i32, i32, f32,
                                             C.POINTER(AdamwHparams), vp, vp]
    lib.psgd_workspace_size.restype = i32
    lib.psgd_workspace_size.argtypes = [i32, i32, i32, i32, C.POINTER(sz)]
    for name in ("psgd_project", "psgd_orthogonalize", "psgd_decompress", "psgd_step"):
        fn = getattr(lib, name)
        fn.restype = i32
        fn.argtypes = [i32, C.POINTER(PsgdMatrix), i32, i32, vp]
    qp = C.POINTER(_Q8Tensor)
    for name, types in (
            ("q8_encode", [vp, i32, i64, i32, i64, qp, vp]),
            ("q8_decode", [qp, i64, i32, i32, vp, i32, i64, vp]),
            ("ln_forward", [vp, i32, i64, i32, i64, vp, vp, f32, vp, i64, vp, vp, qp, vp]),
            ("ln_recompute", [vp, i64, qp, i32, i64, i32, vp, vp, vp, vp, vp, i64, vp]),
            ("ln_workspace_size", [i64, i32, C.POINTER(sz)]),
            ("ln_backward", [vp, i64, vp, i64, qp, i32, i64, i32, vp, vp, vp, vp, i64, vp, i64, vp, vp, i32, vp, sz, vp]),
            ("lin_workspace_size", [i32, i64, i32, i32, i32, C.POINTER(sz)]),
            ("lin_workspace_size_unaligned", [i32, i64, i32, i32, i32, C.POINTER(sz)]),
            ("lin_product_plan", [i32, i64, i32, i32, i32, C.POINTER(_LinPlan)]),
            ("lin_forward", [vp, i64, i32, i64, i32, i32, vp, i64, vp, i32, vp, i64, vp, i64, vp, i64, qp, vp, sz, vp]),
            ("lin_backward_act", [vp, i64, vp, i64, qp, i32, i64, i32, i32, vp, i64, vp]),
            ("lin_backward_input", [vp, i64, i32, i64, i32, i32, vp, i64, i32, vp, i64, qp, vp, i64, vp, sz, vp]),
            ("lin_backward_weight", [vp, i64, vp, i64, qp, i32, i32, i64, i32, i32, vp, i32, i64, vp, i32, vp, sz, vp])):
        fn = getattr(lib, name)
        fn.restype = i32
        fn.argtypes = types
    lib.acsc_stats_enable.restype = i32
    lib.acsc_stats_enable.argtypes = [i32]
    lib.acsc_stats_only.restype = i32
    lib.acsc_stats_only.argtypes = [C.c_char_p]
    lib.acsc_stats_read.restype = i32
    lib.acsc_stats_read.argtypes = [i32, C.c_char_p, sz, C.POINTER(i64), C.POINTER(C.c_double)]
    return lib


lib = _load()

EXPORTED = ("acsc_last_error", "acsc_version", "acsc_stats_enable", "acsc_stats_only", "acsc_stats_read",
            "ac_keep_count", "ac_mask_pack", "ac_unpack_scatter", "ac_mask_pack_batched",
            "ac_unpack_scatter_batched", "sc_workspace_size",
            "sc_build_prior", "sc_correct", "sc_correct_static", "sc_build_prior_batched", "sc_correct_batched",
            "sc_build_subspace_batched", "sc_build_ritz_batched", "sc_build_status",
            "sc_adamw_workspace_size", "sc_correct_adamw_batched",
            "ac_bern_mask", "ac_bern_pack", "ac_bern_unpack",
            "psgd_workspace_size", "psgd_project", "psgd_orthogonalize", "psgd_decompress", "psgd_step",
            "q8_encode", "q8_decode", "ln_forward", "ln_recompute", "ln_workspace_size", "ln_backward",
            "lin_workspace_size", "lin_workspace_size_unaligned", "lin_product_plan", "lin_forward", "lin_backward_act",
            "lin_backward_input", "lin_backward_weight")


def _check(rc: int):
    if rc != 0:
        raise AcscError(rc, lib.acsc_last_error().decode())


def _dt(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return F32
    if t.dtype == torch.bfloat16:
        return BF16
    raise AcscError(ACSC_EDTYPE, f"unsupported dtype {t.dtype}")


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream(stream=None):
    if stream is None:
        # the current stream's handle without the Stream object around it (0.2 us against 2.8 a call)
        return C.c_void_p(torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    return C.c_void_p(stream.cuda_stream)


def _on(stream, fn, *args):
    """fn(*args) on `stream`, if that is not the current one: everything it
    allocates comes from that stream's memory, so it waits for nothing that the
    current stream still does with a block it freed.  What it is given is kept
    from reuse until `stream` has got past the call, what it returns until the
    current stream has got past its use of it."""
    here = torch.cuda.current_stream()
    if stream == here:
        return fn(*args)
    with torch.cuda.stream(stream):
        out = fn(*args)
    _record(args, stream)
    _record(out, here)
    return out


def _record(obj, stream):
    if isinstance(obj, torch.Tensor):
        if obj.is_cuda:
            obj.record_stream(stream)
    elif isinstance(obj, (tuple, list)):
        for o in obj:
            _record(o, stream)


def _need_cuda(*ts):
    for t in ts:
        if t is not None and not t.is_cuda:
            raise AcscError(ACSC_EINVAL, "tensors must live on the GPU")


def _in(t: Optional[torch.Tensor], stream=None) -> Optional[torch.Tensor]:
    """Row-major copy of an input, made on the call's stream, if it is not
    already contiguous."""
    if t is None or t.is_contiguous():
        return t
    return t.contiguous() if stream is None else _on(stream, torch.Tensor.contiguous, t)


def _out(*ts):
    for t in ts:
        if t is not None and not t.is_contiguous():
            raise AcscError(ACSC_EINVAL, "output and in/out tensors must be contiguous")


def acsc_stats_enable(on: bool = True) -> None:
    """Start (resetting the counters) or stop per-kernel event timing."""
    _check(lib.acsc_stats_enable(1 if on else 0))


def acsc_stats_only(tag=None) -> None:
    """Time only the launches of kernel name `tag` (None: every launch)."""
    _check(lib.acsc_stats_only(tag.encode() if tag else None))


def acsc_stats_read() -> dict:
    """{kernel name: (launches, total milliseconds)} of the timed launches."""
    out = {}
    i = 0
    buf = C.create_string_buffer(128)
    n = C.c_int64(0)
    ms = C.c_double(0.0)
    while lib.acsc_stats_read(i, buf, 128, C.byref(n), C.byref(ms)) == 0:
        out[buf.value.decode()] = (n.value, ms.value)
        i += 1
    return out


def make_key(seed: int, layer: int, step: int, microbatch: int, B: int, S: int, H: int) -> MaskKey:
    return MaskKey(seed=seed, step=step, layer=layer, microbatch=microbatch, B=B, S=S, H=H)


def ac_keep_count(H: int, keep: float) -> int:
    k = C.c_int(0)
    _check(lib.ac_keep_count(H, keep, C.byref(k)))
    return k.value


def ac_mask_pack(x: torch.Tensor, K: int, key: MaskKey, vals: Optional[torch.Tensor] = None,
                 idx: Optional[torch.Tensor] = None, with_idx: bool = True, stream=None):
    """x: [rows, H] (row stride x.stride(0)).  Returns (vals [rows, K], idx
    [rows, K] int16 holding uint16 patterns, or None)."""
    if stream is not None:
        return _on(stream, ac_mask_pack, x, K, key, vals, idx, with_idx)
    _need_cuda(x)
    if x.dim() != 2 or x.stride(1) != 1:
        raise AcscError(ACSC_EINVAL, "x must be 2-D with unit column stride")
    rows, H = x.shape
    if vals is None:
        vals = torch.empty(rows, K, dtype=x.dtype, device=x.device)
    if idx is None and with_idx:
        idx = torch.empty(rows, K, dtype=torch.int16, device=x.device)
    _need_cuda(vals, idx)
    _check(lib.ac_mask_pack(_ptr(x), _dt(x), rows, H, x.stride(0), K, C.byref(key), _ptr(vals),
                            _ptr(idx), _stream()))
    return vals, idx


def ac_unpack_scatter(vals: torch.Tensor, H: int, key: MaskKey, scale: float = 1.0,
                      idx: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                      stream=None) -> torch.Tensor:
    """Dense [rows, H] output (or into ``y``, row stride y.stride(0))."""
    if stream is not None:
        return _on(stream, ac_unpack_scatter, vals, H, key, scale, idx, y)
    _need_cuda(vals, idx)
    rows, K = vals.shape
    if y is None:
        y = torch.empty(rows, H, dtype=vals.dtype, device=vals.device)
    _need_cuda(y)
    if y.dim() != 2 or y.stride(1) != 1 or not vals.is_contiguous():
        raise AcscError(ACSC_EINVAL, "vals must be contiguous and y 2-D with unit column stride")
    _check(lib.ac_unpack_scatter(_ptr(vals), _ptr(idx), _dt(vals), rows, H, K, C.byref(key),
                                 float(scale), _ptr(y), y.stride(0), _stream()))
    return y


def _layer_stride(t: torch.Tensor) -> int:
    return t.stride(0) if t.shape[0] > 1 else 0


def ac_mask_pack_batched(x: torch.Tensor, K: int, key: MaskKey, vals: Optional[torch.Tensor] = None,
                         idx_in: Optional[torch.Tensor] = None, idx_out: Optional[torch.Tensor] = None,
                         stream=None) -> torch.Tensor:
    """x: [nlayers, rows, H] (unit column stride; row and layer strides taken
    from the tensor).  Boundary l is keyed with key.layer + l.  Returns vals
    [nlayers, rows, K].  idx_in: [nlayers, rows, K] index lists to pack at
    (no mask evaluated); idx_out: receives the kept positions (int16 holding
    uint16 patterns)."""
    if stream is not None:
        return _on(stream, ac_mask_pack_batched, x, K, key, vals, idx_in, idx_out)
    _need_cuda(x, vals, idx_in, idx_out)
    if x.dim() != 3 or x.stride(2) != 1:
        raise AcscError(ACSC_EINVAL, "x must be [nlayers, rows, H] with unit column stride")
    nl, rows, H = x.shape
    if vals is None:
        vals = torch.empty(nl, rows, K, dtype=x.dtype, device=x.device)
    _need_cuda(vals)
    idx_stride = 0
    for t in (idx_in, idx_out):
        if t is not None:
            if tuple(t.shape) != (nl, rows, K) or t.stride(2) != 1 or t.stride(1) != K:
                raise AcscError(ACSC_EINVAL, "index lists must be [nlayers, rows, K] with contiguous rows")
            idx_stride = _layer_stride(t)
    if tuple(vals.shape) != (nl, rows, K) or vals.stride(2) != 1 or vals.stride(1) != K:
        raise AcscError(ACSC_EINVAL, "vals must be [nlayers, rows, K] with contiguous rows")
    _check(lib.ac_mask_pack_batched(_ptr(x), _dt(x), nl, rows, H, x.stride(1), _layer_stride(x), K, C.byref(key),
                                    _ptr(vals), _layer_stride(vals), _ptr(idx_in), _ptr(idx_out), idx_stride,
                                    _stream()))
    return vals


def ac_unpack_scatter_batched(vals: torch.Tensor, H: int, key: MaskKey, scale: float = 1.0,
                              idx_in: Optional[torch.Tensor] = None, idx_out: Optional[torch.Tensor] = None,
                              y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """vals: [nlayers, rows, K].  Returns (or fills) y [nlayers, rows, H].
    idx_in: transmitted or kept index lists; idx_out: receives the positions
    rebuilt from the key."""
    if stream is not None:
        return _on(stream, ac_unpack_scatter_batched, vals, H, key, scale, idx_in, idx_out, y)
    _need_cuda(vals, idx_in, idx_out)
    if vals.dim() != 3 or vals.stride(2) != 1 or vals.stride(1) != vals.shape[2]:
        raise AcscError(ACSC_EINVAL, "vals must be [nlayers, rows, K] with contiguous rows")
    nl, rows, K = vals.shape
    if y is None:
        y = torch.empty(nl, rows, H, dtype=vals.dtype, device=vals.device)
    _need_cuda(y)
    if y.dim() != 3 or y.stride(2) != 1 or tuple(y.shape) != (nl, rows, H):
        raise AcscError(ACSC_EINVAL, "y must be [nlayers, rows, H] with unit column stride")
    idx_stride = 0
    for t in (idx_in, idx_out):
        if t is not None:
            if tuple(t.shape) != (nl, rows, K) or t.stride(2) != 1 or t.stride(1) != K:
                raise AcscError(ACSC_EINVAL, "index lists must be [nlayers, rows, K] with contiguous rows")
            idx_stride = _layer_stride(t)
    _check(lib.ac_unpack_scatter_batched(_ptr(vals), _layer_stride(vals), _dt(vals), nl, rows, H, K, C.byref(key),
                                         _ptr(idx_in), _ptr(idx_out), idx_stride, float(scale), _ptr(y), y.stride(1),
                                         _layer_stride(y), _stream()))
    return y


def ac_bern_mask(rows: int, H: int, keep: float, key: MaskKey, device="cuda", stream=None):
    """The Bernoulli mask of a [rows, H] tensor: (row_ptr int64 [rows + 1],
    bits int32 [rows, ceil(H / 32)] holding uint32 patterns)."""
    if stream is not None:
        return _on(stream, ac_bern_mask, rows, H, keep, key, device)
    row_ptr = torch.empty(rows + 1, dtype=torch.int64, device=device)
    bits = torch.empty(max(rows, 1), (H + 31) // 32, dtype=torch.int32, device=device)[:rows]
    _check(lib.ac_bern_mask(rows, H, float(keep), C.byref(key), _ptr(row_ptr), _ptr(bits), _stream()))
    return row_ptr, bits


def ac_bern_pack(x: torch.Tensor, row_ptr: torch.Tensor, bits: torch.Tensor, nnz: Optional[int] = None,
                 with_idx: bool = True, stream=None):
    """Packed values [nnz] (and uint16 indices as int16, or None) of x [rows, H]
    under the mask (row_ptr, bits).  nnz defaults to row_ptr[-1] (a host
    read, which synchronises)."""
    if stream is not None:
        return _on(stream, ac_bern_pack, x, row_ptr, bits, nnz, with_idx)
    _need_cuda(x, row_ptr, bits)
    if x.dim() != 2 or x.stride(1) != 1:
        raise AcscError(ACSC_EINVAL, "x must be 2-D with unit column stride")
    rows, H = x.shape
    if nnz is None:
        nnz = int(row_ptr[-1].item())
    vals = torch.empty(max(nnz, 1), dtype=x.dtype, device=x.device)[:nnz]
    idx = torch.empty(max(nnz, 1), dtype=torch.int16, device=x.device)[:nnz] if with_idx else None
    _check(lib.ac_bern_pack(_ptr(x), _dt(x), rows, H, x.stride(0), _ptr(row_ptr), _ptr(bits), _ptr(vals),
                            _ptr(idx), nnz, _stream()))
    return vals, idx


def ac_bern_unpack(vals: torch.Tensor, H: int, row_ptr: torch.Tensor, bits: torch.Tensor, scale: float = 1.0,
                   y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Dense [rows, H]: scale * value at the kept entries, +0 elsewhere."""
    if stream is not None:
        return _on(stream, ac_bern_unpack, vals, H, row_ptr, bits, scale, y)
    _need_cuda(vals, row_ptr, bits)
    rows = row_ptr.numel() - 1
    if y is None:
        y = torch.empty(rows, H, dtype=vals.dtype, device=vals.device)
    _need_cuda(y)
    if y.dim() != 2 or y.stride(1) != 1 or not vals.is_contiguous():
        raise AcscError(ACSC_EINVAL, "vals must be contiguous and y 2-D with unit column stride")
    _check(lib.ac_bern_unpack(_ptr(vals), _dt(vals), rows, H, _ptr(row_ptr), _ptr(bits), vals.numel(),
                              float(scale), _ptr(y), y.stride(0), _stream()))
    return y


def sc_workspace_size(m: int, n: int, r: int, oversample: int, dtype: torch.dtype) -> int:
    b = C.c_size_t(0)
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(lib.sc_workspace_size(m, n, r, oversample, code, C.byref(b)))
    return b.value


def workspace(m: int, n: int, r: int, oversample: int, dtype: torch.dtype, device="cuda"):
    nbytes = sc_workspace_size(m, n, r, oversample, dtype)
    return torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)


def sc_build_prior(G_anc: Optional[torch.Tensor], M: torch.Tensor, r: int, beta: float,
                   tau: float, oversample: int, power_iters: int, seed: int = 0,
                   V_warm: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                   out=None, dtype: Optional[torch.dtype] = None, stream=None):
    """EMA of G_anc into M (fp32, in place), then (U, s, V, d).  Returns them."""
    if stream is not None:
        return _on(stream, sc_build_prior, G_anc, M, r, beta, tau, oversample, power_iters, seed, V_warm, ws, out, dtype)
    _need_cuda(G_anc, M, V_warm)
    G_anc, V_warm = _in(G_anc), _in(V_warm)
    _out(M)
    m, n = M.shape
    dt = dtype if dtype is not None else (G_anc.dtype if G_anc is not None else torch.float32)
    if out is None:
        out = (torch.empty(m, r, device=M.device), torch.empty(r, device=M.device),
               torch.empty(n, r, device=M.device), torch.empty(r, device=M.device))
    U, s, V, d = out
    _out(U, s, V, d)
    if ws is None:
        ws = workspace(m, n, r, oversample, dt, M.device)
    code = BF16 if dt == torch.bfloat16 else F32
    _check(lib.sc_build_prior(_ptr(G_anc), code, _ptr(M), m, n, float(beta), r, oversample,
                              power_iters, float(tau), _ptr(V_warm), seed, _ptr(U), _ptr(s),
                              _ptr(V), _ptr(d), _ptr(ws), ws.numel(), _stream()))
    return U, s, V, d


def sc_correct(G: torch.Tensor, U: torch.Tensor, d: torch.Tensor, V: torch.Tensor, alpha: float,
               out: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
               stream=None) -> torch.Tensor:
    """G_proj = alpha G + (1 - alpha) U diag(d) U^T G V diag(d) V^T."""
    if stream is not None:
        return _on(stream, sc_correct, G, U, d, V, alpha, out, ws)
    _need_cuda(G, U, d, V, out)
    G, U, d, V = _in(G), _in(U), _in(d), _in(V)
    _out(out)
    m, n = G.shape
    r = U.shape[1]
    if out is None:
        out = torch.empty_like(G)
    if ws is None:
        ws = workspace(m, n, r, 0, G.dtype, G.device)
    _check(lib.sc_correct(_ptr(G), _dt(G), m, n, _ptr(U), _ptr(d), _ptr(V), r, float(alpha),
                          _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out


SC_STATIC_SCRATCH_BYTES = 96 * 1024 * 1024


def sc_correct_static(G: torch.Tensor, U: torch.Tensor, d: torch.Tensor, V: torch.Tensor, alpha: float,
                      out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """sc_correct on the library's own device scratch (no workspace; for
    callers that cannot allocate).  ``out`` must be given by a caller that
    cannot allocate; calls that overlap on one GPU race."""
    if stream is not None:
        return _on(stream, sc_correct_static, G, U, d, V, alpha, out)
    _need_cuda(G, U, d, V, out)
    for t in (G, U, d, V):
        if not t.is_contiguous():
            raise AcscError(ACSC_EINVAL, "G, U, d, V must be contiguous (no copies are made)")
    _out(out)
    m, n = G.shape
    r = U.shape[1]
    if out is None:
        out = torch.empty_like(G)
    _check(lib.sc_correct_static(_ptr(G), _dt(G), m, n, _ptr(U), _ptr(d), _ptr(V), r, float(alpha), _ptr(out),
                                 _stream()))
    return out


def _p(t):
    return None if t is None else t.data_ptr()


def sc_build_prior_batched(items, r: int, beta: float, tau: float, oversample: int,
                           power_iters: int, seed: int = 0, dtype: torch.dtype = torch.bfloat16,
                           stream=None):
    """items: list of dicts with G_anc (or None), M, out=(U, s, V, d), ws, and
    optionally V_warm.  Matrix i starts from the random block of seed + i."""
    _build_batched(lib.sc_build_prior_batched, items, r, beta, tau, oversample, power_iters, seed, dtype, stream)


def sc_build_subspace_batched(items, r: int, beta: float, tau: float, oversample: int,
                              power_iters: int, seed: int = 0, dtype: torch.dtype = torch.bfloat16,
                              stream=None):
    """First phase of sc_build_prior_batched (EMA, power passes, Z = M^T Q);
    the same arguments.  Follow it with sc_build_ritz_batched."""
    _build_batched(lib.sc_build_subspace_batched, items, r, beta, tau, oversample, power_iters, seed, dtype,
                   stream)


def sc_build_ritz_batched(items, r: int, beta: float, tau: float, oversample: int,
                          power_iters: int, seed: int = 0, dtype: torch.dtype = torch.bfloat16,
                          stream=None):
    """Second phase of sc_build_prior_batched (Rayleigh-Ritz on Z: U, s, V, d);
    the same arguments and workspaces as the sc_build_subspace_batched call
    it follows, whose matrices may come in several such calls."""
    _build_batched(lib.sc_build_ritz_batched, items, r, beta, tau, oversample, power_iters, seed, dtype, stream)


def _build_batched(fn, items, r, beta, tau, oversample, power_iters, seed, dtype, stream):
    arr = (ScMatrix * max(len(items), 1))()
    keep = []
    for i, it in enumerate(items):
        G, M, (U, s, V, d), ws = _in(it.get("G_anc"), stream), it["M"], it["out"], it["ws"]
        Vw = _in(it.get("V_warm"), stream)
        _need_cuda(G, M, U, s, V, d, ws, Vw)
        _out(M, U, s, V, d)
        keep += [G, Vw]
        m, n = M.shape
        arr[i] = ScMatrix(_p(G), _p(M), m, n, _p(U), _p(s), _p(V), _p(d), _p(Vw), None, _p(ws),
                          ws.numel())
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(fn(len(items), arr, code, float(beta), r, oversample, power_iters, float(tau), seed, _stream(stream)))


def sc_build_status(workspaces, stream=None):
    """Synchronise and read the status the last build left in each workspace:
    a list of (sweeps, residual) per workspace.  Raises AcscError with code
    ACSC_ENOCONV when a build stopped at its sweep cap above tolerance or ran
    its Rayleigh-Ritz phase without a subspace phase."""
    n = len(workspaces)
    arr = (ScMatrix * max(n, 1))()
    for i, ws in enumerate(workspaces):
        _need_cuda(ws)
        arr[i] = ScMatrix(None, None, 0, 0, None, None, None, None, None, None, _p(ws), ws.numel())
    sweeps = (C.c_int * max(n, 1))()
    res = (C.c_float * max(n, 1))()
    rc = lib.sc_build_status(n, arr, sweeps, res, _stream(stream))
    out = [(sweeps[i], res[i]) for i in range(n)]
    if rc != 0:
        err = AcscError(rc, lib.acsc_last_error().decode())
        err.status = out
        raise err
    return out


def sc_correct_batched(items, r: int, alpha: float, dtype: torch.dtype = torch.bfloat16,
                       stream=None):
    """items: list of dicts with G, prior=(U, d, V), out (G_proj) and ws."""
    arr = (ScMatrix * max(len(items), 1))()
    keep = []
    for i, it in enumerate(items):
        G, (U, d, V), out, ws = _in(it["G"], stream), it["prior"], it["out"], it["ws"]
        U, d, V = _in(U, stream), _in(d, stream), _in(V, stream)
        _need_cuda(G, U, d, V, out, ws)
        _out(out)
        keep += [G, U, d, V]
        m, n = G.shape
        arr[i] = ScMatrix(_p(G), None, m, n, _p(U), _p(d), _p(V), _p(d), None, _p(out), _p(ws),
                          ws.numel())
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(lib.sc_correct_batched(len(items), arr, code, r, float(alpha), _stream(stream)))


def sc_adamw_workspace_size(m: int, n: int, r: int, dtype: torch.dtype) -> int:
    b = C.c_size_t(0)
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(lib.sc_adamw_workspace_size(m, n, r, code, C.byref(b)))
    return b.value


def sc_correct_adamw_batched(items, r: int, alpha: float, lr: float, beta1: float = 0.9,
                             beta2: float = 0.999, eps: float = 1e-8, weight_decay: float = 0.0,
                             step: int = 1, max_norm: float = 0.0, dtype: torch.dtype = torch.bfloat16,
                             norm_out: Optional[torch.Tensor] = None, stream=None):
    """items: list of dicts with G, prior=(U, d, V), ws and state=(W, m1, m2)
    (fp32, updated in place).  norm_out: optional fp32 device scalar that
    receives the global norm of the G_proj before clipping."""
    arr = (ScMatrix * max(len(items), 1))()
    st = (AdamwState * max(len(items), 1))()
    keep = []
    for i, it in enumerate(items):
        G, (U, d, V), ws, (W, m1, m2) = _in(it["G"], stream), it["prior"], it["ws"], it["state"]
        U, d, V = _in(U, stream), _in(d, stream), _in(V, stream)
        _need_cuda(G, U, d, V, ws, W, m1, m2, norm_out)
        _out(W, m1, m2)
        for t in (W, m1, m2):
            if t.dtype != torch.float32 or tuple(t.shape) != tuple(G.shape):
                raise AcscError(ACSC_EINVAL, "W, m1, m2 must be fp32 tensors of G's shape")
        keep += [G, U, d, V]
        m, n = G.shape
        arr[i] = ScMatrix(_p(G), None, m, n, _p(U), _p(d), _p(V), _p(d), None, None, _p(ws), ws.numel())
        st[i] = AdamwState(_p(W), _p(m1), _p(m2))
    hp = AdamwHparams(float(lr), float(beta1), float(beta2), float(eps), float(weight_decay), int(step),
                      float(max_norm))
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(lib.sc_correct_adamw_batched(len(items), arr, st, code, r, float(alpha), C.byref(hp),
                                        _ptr(norm_out), _stream(stream)))


def psgd_workspace_size(m: int, n: int, r: int, dtype: torch.dtype) -> int:
    b = C.c_size_t(0)
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(lib.psgd_workspace_size(m, n, r, code, C.byref(b)))
    return b.value


def psgd_workspace(m: int, n: int, r: int, dtype: torch.dtype, device="cuda"):
    return torch.empty(max(psgd_workspace_size(m, n, r, dtype), 256), dtype=torch.uint8, device=device)


def _psgd(name: str, items, r: int, dtype: torch.dtype, stream):
    arr = (PsgdMatrix * max(len(items), 1))()
    keep = []
    for i, it in enumerate(items):
        G, E, P, Q, out, ws = _in(it.get("G"), stream), it["E"], it["P"], it["Q"], it.get("out"), it["ws"]
        _need_cuda(G, E, P, Q, out, ws)
        _out(E, P, Q, out)
        for t, shape in ((E, None), (P, (E.shape[0], r)), (Q, (E.shape[1], r))):
            if t.dtype != torch.float32 or (shape is not None and tuple(t.shape) != shape):
                raise AcscError(ACSC_EINVAL, "E [m, n], P [m, r], Q [n, r] must be fp32")
        keep.append(G)
        m, n = E.shape
        arr[i] = PsgdMatrix(_p(G), _p(E), _p(P), _p(Q), _p(out), m, n, _p(ws), ws.numel())
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(getattr(lib, name)(len(items), arr, code, r, _stream(stream)))


def psgd_project(items, r: int, dtype: torch.dtype = torch.bfloat16, stream=None):
    """items: dicts with G, E, P, Q, ws (out unused): E <- E + G, P <- E Q."""
    _psgd("psgd_project", items, r, dtype, stream)


def psgd_orthogonalize(items, r: int, dtype: torch.dtype = torch.bfloat16, stream=None):
    """P <- orth(P), Q <- M^T P (M held in E and in the workspace)."""
    _psgd("psgd_orthogonalize", items, r, dtype, stream)


def psgd_decompress(items, r: int, dtype: torch.dtype = torch.bfloat16, stream=None):
    """out <- P Q^T (in dtype), E <- M - out."""
    _psgd("psgd_decompress", items, r, dtype, stream)


def psgd_step(items, r: int, dtype: torch.dtype = torch.bfloat16, stream=None):
    """The three phases on one worker (items: dicts with G, E, P, Q, out, ws)."""
    _psgd("psgd_step", items, r, dtype, stream)


Q8_GROUP = 128
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
LIN_FORWARD, LIN_BACKWARD_INPUT, LIN_BACKWARD_WEIGHT = 0, 1, 2


# Small calls are bound by what these few lines cost on the host (a launch
# takes 5 us): attributes are read once, pointers go as plain integers, sizes
# that depend on shapes alone are kept.

def _act(act: str) -> int:
    code = ACTS.get(act)
    if code is None:
        raise AcscError(ACSC_EINVAL, f"unknown activation {act!r}: one of {', '.join(ACTS)}")
    return code


def _raw_stream() -> int:
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _rows(t: torch.Tensor, shape, dtype: torch.dtype, name: str) -> int:
    """The row stride of a [rows, cols] tensor with unit column stride."""
    if not t.is_cuda:
        raise AcscError(ACSC_EINVAL, "tensors must live on the GPU")
    if t.shape != shape:
        raise AcscError(ACSC_EINVAL, f"{name} must be {list(shape)}, not {list(t.shape)}")
    if t.dtype is not dtype:
        raise AcscError(ACSC_EDTYPE, f"{name} must be {dtype}, not {t.dtype}")
    ld, unit = t.stride()
    if unit != 1 and shape[1] > 1:
        raise AcscError(ACSC_EINVAL, f"{name} must have unit column stride")
    # the stride of a single row, or of none, means nothing
    return ld if shape[0] > 1 else max(shape[1], 1)


def _vec(t: torch.Tensor, n: int, dtype: torch.dtype, name: str) -> int:
    """The address of a contiguous [n] tensor."""
    if not t.is_cuda:
        raise AcscError(ACSC_EINVAL, "tensors must live on the GPU")
    if t.shape != (n,) or not t.is_contiguous():
        raise AcscError(ACSC_EINVAL, f"{name} must be [{n}] and contiguous")
    if t.dtype is not dtype:
        raise AcscError(ACSC_EDTYPE, f"{name} must be {dtype}, not {t.dtype}")
    return t.data_ptr()


def _two_d(t: torch.Tensor, name: str):
    if t.dim() != 2:
        raise AcscError(ACSC_EINVAL, f"{name} must be 2-D")
    return t.shape


def _q8_new(rows: int, H: int, device) -> Q8:
    return Q8(torch.empty((rows, H), dtype=torch.int8, device=device),
              torch.empty((rows, -(-H // Q8_GROUP)), dtype=torch.float32, device=device))


def _q8_ref(q: Q8, rows: int, H: int):
    codes, scales = q
    ldc = _rows(codes, (rows, H), torch.int8, "codes")
    lds = _rows(scales, (rows, -(-H // Q8_GROUP)), torch.float32, "scales")
    return C.byref(_Q8Tensor(codes.data_ptr(), scales.data_ptr(), ldc, lds))


def _kept(src: Union[torch.Tensor, Q8, None], shape, dtype: torch.dtype, name: str):
    """(pointer, row stride, checkpoint) of a tensor or its checkpoint."""
    if src is None:
        return None, 0, None
    if isinstance(src, Q8):
        return None, 0, _q8_ref(src, shape[0], shape[1])
    ld = _rows(src, shape, dtype, name)
    return src.data_ptr(), ld, None


def _ws(nbytes: int, ws: Optional[torch.Tensor], device):
    """(address, bytes, what keeps it alive) of a workspace: the given one, or a new one."""
    if ws is None:
        if not nbytes:
            return None, 0, None
        ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return ws.data_ptr(), nbytes, ws
    _need_cuda(ws)
    return ws.data_ptr(), ws.numel() * ws.element_size(), ws


@functools.lru_cache(maxsize=1024)
def _lin_bytes(aligned: bool, op: int, rows: int, n_in: int, n_out: int, dtype: torch.dtype) -> int:
    return (lin_workspace_size if aligned else lin_workspace_size_unaligned)(op, rows, n_in, n_out, dtype)


@functools.lru_cache(maxsize=1024)
def _ln_bytes(rows: int, H: int) -> int:
    return ln_workspace_size(rows, H)


def q8_encode(x: torch.Tensor, q: Optional[Q8] = None, stream=None) -> Q8:
    """The 8-bit checkpoint of x [rows, H] (row stride x.stride(0))."""
    if stream is not None:
        return _on(stream, q8_encode, x, q)
    rows, H = _two_d(x, "x")
    dt, ld = _dt(x), _rows(x, x.shape, x.dtype, "x")
    if q is None:
        q = _q8_new(rows, H, x.device)
    rc = lib.q8_encode(x.data_ptr(), dt, rows, H, ld, _q8_ref(q, rows, H), _raw_stream())
    if rc:
        _check(rc)
    return q


def q8_decode(q: Q8, dtype: torch.dtype, act: str = "none", y: Optional[torch.Tensor] = None,
              stream=None) -> torch.Tensor:
    """act(values of q) [rows, H], rounded once to dtype."""
    if stream is not None:
        return _on(stream, q8_decode, q, dtype, act, y)
    rows, H = _two_d(q.codes, "codes")
    if y is None:
        y = torch.empty((rows, H), dtype=dtype, device=q.codes.device)
    ld = _rows(y, (rows, H), dtype, "y")
    rc = lib.q8_decode(_q8_ref(q, rows, H), rows, H, _act(act), y.data_ptr(), _dt(y), ld, _raw_stream())
    if rc:
        _check(rc)
    return y


def ln_forward(x: torch.Tensor, gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
               eps: float = 1e-5, checkpoint: bool = False, y: Optional[torch.Tensor] = None, stream=None):
    """Layer norm of the rows of x [rows, H]: (y, mean [rows], rstd [rows], q),
    q the 8-bit checkpoint of x if asked for, else None."""
    if stream is not None:
        return _on(stream, ln_forward, x, gamma, beta, eps, checkpoint, y)
    shape = rows, H = _two_d(x, "x")
    dtype, dev = x.dtype, x.device
    ld = _rows(x, shape, dtype, "x")
    pg = None if gamma is None else _vec(gamma, H, dtype, "gamma")
    pb = None if beta is None else _vec(beta, H, dtype, "beta")
    if y is None:
        y, ldy = torch.empty((rows, H), dtype=dtype, device=dev), max(H, 1)
    else:
        ldy = _rows(y, shape, dtype, "y")
    mean = torch.empty(rows, dtype=torch.float32, device=dev)
    rstd = torch.empty(rows, dtype=torch.float32, device=dev)
    q = _q8_new(rows, H, dev) if checkpoint else None
    rc = lib.ln_forward(x.data_ptr(), _dt(x), rows, H, ld, pg, pb, eps, y.data_ptr(), ldy, mean.data_ptr(),
                        rstd.data_ptr(), None if q is None else _q8_ref(q, rows, H), _raw_stream())
    if rc:
        _check(rc)
    return y, mean, rstd, q


def ln_recompute(src: Union[torch.Tensor, Q8], mean: torch.Tensor, rstd: torch.Tensor,
                 gamma: Optional[torch.Tensor] = None, beta: Optional[torch.Tensor] = None,
                 dtype: torch.dtype = torch.bfloat16, y: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """ln_forward's y again from x or its checkpoint and the kept statistics."""
    if stream is not None:
        return _on(stream, ln_recompute, src, mean, rstd, gamma, beta, dtype, y)
    rows, H = _two_d(src.codes if isinstance(src, Q8) else src, "src")
    p, ld, q = _kept(src, (rows, H), dtype, "src")
    pm, pr = _vec(mean, rows, torch.float32, "mean"), _vec(rstd, rows, torch.float32, "rstd")
    pg = None if gamma is None else _vec(gamma, H, dtype, "gamma")
    pb = None if beta is None else _vec(beta, H, dtype, "beta")
    if y is None:
        y = torch.empty((rows, H), dtype=dtype, device=mean.device)
    ldy = _rows(y, (rows, H), dtype, "y")
    _check(lib.ln_recompute(p, ld, q, _dt(y), rows, H, pm, pr, pg, pb, y.data_ptr(), ldy, _raw_stream()))
    return y


def ln_workspace_size(rows: int, H: int) -> int:
    b = C.c_size_t(0)
    _check(lib.ln_workspace_size(rows, H, C.byref(b)))
    return b.value


def ln_backward(dy: torch.Tensor, src: Union[torch.Tensor, Q8], mean: torch.Tensor, rstd: torch.Tensor,
                gamma: Optional[torch.Tensor] = None, add: Optional[torch.Tensor] = None,
                dx: Optional[torch.Tensor] = None, dgamma: Optional[torch.Tensor] = None,
                dbeta: Optional[torch.Tensor] = None, accumulate: bool = False, ws: Optional[torch.Tensor] = None,
                stream=None, weights: bool = True):
    """(dx, dgamma, dbeta) of ln_forward from x or its checkpoint; add: the
    gradient that reaches x past the norm.  dgamma, dbeta: fp32 [H]; with
    accumulate they are given and added to; without weights they are not
    formed, and None."""
    if stream is not None:
        return _on(stream, ln_backward, dy, src, mean, rstd, gamma, add, dx, dgamma, dbeta, accumulate, ws, None, weights)
    shape = rows, H = _two_d(dy, "dy")
    dtype, dev = dy.dtype, dy.device
    lddy = _rows(dy, shape, dtype, "dy")
    p, ld, q = _kept(src, shape, dtype, "src")
    pa, ldadd = (None, 0) if add is None else (add.data_ptr(), _rows(add, shape, dtype, "add"))
    if accumulate and (dgamma is None or dbeta is None):
        raise AcscError(ACSC_EINVAL, "accumulate needs dgamma and dbeta")
    if dx is None:
        dx, lddx = torch.empty((rows, H), dtype=dtype, device=dev), max(H, 1)
    else:
        lddx = _rows(dx, shape, dtype, "dx")
    pdg = pdb = wp = keep = None
    wn = 0
    if weights:
        if dgamma is None:
            dgamma = torch.empty(H, dtype=torch.float32, device=dev)
        if dbeta is None:
            dbeta = torch.empty(H, dtype=torch.float32, device=dev)
        pdg, pdb = _vec(dgamma, H, torch.float32, "dgamma"), _vec(dbeta, H, torch.float32, "dbeta")
        wp, wn, keep = _ws(_ln_bytes(rows, H), ws, dev)
    elif dgamma is not None or dbeta is not None:
        raise AcscError(ACSC_EINVAL, "dgamma and dbeta are given, but not wanted")
    pm, pr = _vec(mean, rows, torch.float32, "mean"), _vec(rstd, rows, torch.float32, "rstd")
    pg = None if gamma is None else _vec(gamma, H, dtype, "gamma")
    rc = lib.ln_backward(dy.data_ptr(), lddy, p, ld, q, _dt(dy), rows, H, pm, pr, pg, pa, ldadd, dx.data_ptr(), lddx,
                         pdg, pdb, int(accumulate), wp, wn, _raw_stream())
    if rc:
        _check(rc)
    return dx, dgamma, dbeta


def lin_workspace_size(op: int, rows: int, n_in: int, n_out: int, dtype: torch.dtype) -> int:
    """Bytes for one product (LIN_FORWARD, LIN_BACKWARD_INPUT, LIN_BACKWARD_WEIGHT) of a linear layer whose
    operands have row strides under 2^21 and, in bf16, are 4-byte aligned with even strides."""
    b = C.c_size_t(0)
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(lib.lin_workspace_size(op, rows, n_in, n_out, code, C.byref(b)))
    return b.value


def lin_workspace_size_unaligned(op: int, rows: int, n_in: int, n_out: int, dtype: torch.dtype) -> int:
    """The same for operands of any alignment and stride."""
    b = C.c_size_t(0)
    code = BF16 if dtype == torch.bfloat16 else F32
    _check(lib.lin_workspace_size_unaligned(op, rows, n_in, n_out, code, C.byref(b)))
    return b.value


def lin_product_plan(op: int, rows: int, n_in: int, n_out: int, dtype: torch.dtype) -> LinPlan:
    """How that product runs, for operands as in lin_workspace_size."""
    p = _LinPlan()
    _check(lib.lin_product_plan(op, rows, n_in, n_out, BF16 if dtype == torch.bfloat16 else F32, C.byref(p)))
    return LinPlan(p.tile_rows, p.tile_cols, p.whole, p.cut, p.pieces)


def _lin_ws(op: int, rows: int, n_in: int, n_out: int, a, lda: int, b, ldb: int, ws: Optional[torch.Tensor]):
    """A workspace for a product of operands a and b (their row strides; b may
    be None), unless one is given."""
    if ws is not None:
        return _ws(0, ws, a.device)
    aligned = lda < 1 << 21 and (b is None or ldb < 1 << 21)
    if aligned and a.dtype is torch.bfloat16:
        aligned = not ((lda | a.data_ptr() >> 1) & 1) and (b is None or not ((ldb | b.data_ptr() >> 1) & 1))
    return _ws(_lin_bytes(aligned, op, rows, n_in, n_out, a.dtype), None, a.device)


def lin_forward(x: torch.Tensor, W: torch.Tensor, bias: Optional[torch.Tensor] = None, act: str = "none",
                residual: Optional[torch.Tensor] = None, keep: Optional[str] = None, y: Optional[torch.Tensor] = None,
                ws: Optional[torch.Tensor] = None, stream=None):
    """y = act(x W^T + bias) + residual for x [rows, n_in], W [n_out, n_in]:
    (y, kept), kept the pre-activation if keep is "z", its 8-bit checkpoint if
    keep is "q8", else None."""
    if stream is not None:
        return _on(stream, lin_forward, x, W, bias, act, residual, keep, y, ws)
    rows, n_in = _two_d(x, "x")
    n_out = _two_d(W, "W")[0]
    dtype, dev = x.dtype, x.device
    ldx, ldw = _rows(x, (rows, n_in), dtype, "x"), _rows(W, (n_out, n_in), dtype, "W")
    pb = None if bias is None else _vec(bias, n_out, dtype, "bias")
    shape = (rows, n_out)
    pr, ldr = (None, 0) if residual is None else (residual.data_ptr(), _rows(residual, shape, dtype, "residual"))
    if y is None:
        y, ldy = torch.empty(shape, dtype=dtype, device=dev), n_out
    else:
        ldy = _rows(y, shape, dtype, "y")
    z = q = pz = pq = None
    if keep == "z":
        z = torch.empty(shape, dtype=dtype, device=dev)
        pz = z.data_ptr()
    elif keep == "q8":
        q = _q8_new(rows, n_out, dev)
        pq = _q8_ref(q, rows, n_out)
    elif keep is not None:
        raise AcscError(ACSC_EINVAL, f"keep must be None, 'z' or 'q8', not {keep!r}")
    wp, wn, hold = _lin_ws(LIN_FORWARD, rows, n_in, n_out, x, ldx, W, ldw, ws)
    rc = lib.lin_forward(x.data_ptr(), ldx, _dt(x), rows, n_in, n_out, W.data_ptr(), ldw, pb, _act(act), pr, ldr,
                         y.data_ptr(), ldy, pz, n_out, pq, wp, wn, _raw_stream())
    if rc:
        _check(rc)
    return y, (z if q is None else q)


def lin_backward_act(dy: torch.Tensor, z: Union[torch.Tensor, Q8], act: str, dz: Optional[torch.Tensor] = None,
                     stream=None) -> torch.Tensor:
    """dz = dy act'(z) from the kept pre-activation or its checkpoint."""
    if stream is not None:
        return _on(stream, lin_backward_act, dy, z, act, dz)
    shape = rows, n = _two_d(dy, "dy")
    ld = _rows(dy, shape, dy.dtype, "dy")
    p, ldz, q = _kept(z, shape, dy.dtype, "z")
    if dz is None:
        dz, lddz = torch.empty((rows, n), dtype=dy.dtype, device=dy.device), max(n, 1)
    else:
        lddz = _rows(dz, shape, dy.dtype, "dz")
    rc = lib.lin_backward_act(dy.data_ptr(), ld, p, ldz, q, _dt(dy), rows, n, _act(act), dz.data_ptr(), lddz,
                              _raw_stream())
    if rc:
        _check(rc)
    return dz


def lin_backward_input(dz: torch.Tensor, W: torch.Tensor, act: str = "none",
                       z: Union[torch.Tensor, Q8, None] = None, dx: Optional[torch.Tensor] = None,
                       ws: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """dx = dz W; with act, (dz W) act'(z) from the pre-activation z [rows,
    n_in] that the layer before kept, or its checkpoint."""
    if stream is not None:
        return _on(stream, lin_backward_input, dz, W, act, z, dx, ws)
    rows, n_out = _two_d(dz, "dz")
    n_in = _two_d(W, "W")[1]
    dtype, dev = dz.dtype, dz.device
    lddz, ldw = _rows(dz, (rows, n_out), dtype, "dz"), _rows(W, (n_out, n_in), dtype, "W")
    p, ldz, q = _kept(z, (rows, n_in), dtype, "z")
    if dx is None:
        dx, lddx = torch.empty((rows, n_in), dtype=dtype, device=dev), n_in
    else:
        lddx = _rows(dx, (rows, n_in), dtype, "dx")
    wp, wn, hold = _lin_ws(LIN_BACKWARD_INPUT, rows, n_in, n_out, dz, lddz, W, ldw, ws)
    rc = lib.lin_backward_input(dz.data_ptr(), lddz, _dt(dz), rows, n_in, n_out, W.data_ptr(), ldw, _act(act), p, ldz, q,
                                dx.data_ptr(), lddx, wp, wn, _raw_stream())
    if rc:
        _check(rc)
    return dx


def lin_backward_weight(dz: torch.Tensor, x: Union[torch.Tensor, Q8], act: str = "none",
                        dw_dtype: Optional[torch.dtype] = None, bias: bool = True, dW: Optional[torch.Tensor] = None,
                        db: Optional[torch.Tensor] = None, accumulate: bool = False, ws: Optional[torch.Tensor] = None,
                        stream=None):
    """(dW [n_out, n_in] of dw_dtype (dz's by default), db fp32 [n_out] or None)
    from dz [rows, n_out] and the layer's input act(x), x [rows, n_in] or its
    checkpoint.  With accumulate, dW (and db, unless bias is False) are given
    and added to."""
    if stream is not None:
        return _on(stream, lin_backward_weight, dz, x, act, dw_dtype, bias, dW, db, accumulate, ws)
    rows, n_out = _two_d(dz, "dz")
    n_in = _two_d(x.codes if isinstance(x, Q8) else x, "x")[1]
    dtype, dev = dz.dtype, dz.device
    lddz = _rows(dz, (rows, n_out), dtype, "dz")
    p, ldx, q = _kept(x, (rows, n_in), dtype, "x")
    if accumulate and (dW is None or (bias and db is None)):
        raise AcscError(ACSC_EINVAL, "accumulate needs dW and db")
    if dW is None:
        dW, lddw = torch.empty((n_out, n_in), dtype=dw_dtype or dtype, device=dev), n_in
    else:
        lddw = _rows(dW, (n_out, n_in), dw_dtype or dW.dtype, "dW")
    if db is None and bias:
        db = torch.empty(n_out, dtype=torch.float32, device=dev)
    pdb = None if db is None else _vec(db, n_out, torch.float32, "db")
    code = _act(act)
    # the activation is recomputed into the workspace: no operand of the caller's
    wp, wn, hold = _lin_ws(LIN_BACKWARD_WEIGHT, rows, n_in, n_out, dz, lddz, None if q is not None or code else x, ldx, ws)
    rc = lib.lin_backward_weight(dz.data_ptr(), lddz, p, ldx, q, code, _dt(dz), rows, n_in, n_out, dW.data_ptr(), _dt(dW),
                                 lddw, pdb, int(accumulate), wp, wn, _raw_stream())
    if rc:
        _check(rc)
    return dW, db
