"""ctypes binding of the layer operators of libtsenor.so (declared in include/tsenor_layer.h): quantisation into 8-bit
floating point, root-mean-square norm, 8-bit product, gradient clipping.

As in ``binding``: argument marshalling only, ``make_*`` describes a call once (no copies; the tensors must outlive it), the
function named like the C entry point enqueues it as often as wanted, on the current stream of the GPU that the tensors are on
(on ``stream`` if given, which has to be one of that GPU).
"""
from __future__ import annotations

import ctypes
from dataclasses import dataclass
from typing import Any

from .binding import TSENOR_BF16, TSENOR_F32, TSENOR_OK, TsenorError, current_device, current_stream, load

TSENOR_SCALE_BLOCK = 128


class tsenor_scaled(ctypes.Structure):
    _fields_ = [
        ("values", ctypes.c_void_p),
        ("scales", ctypes.c_void_p),
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("ld", ctypes.c_int64),
        ("scale_ld", ctypes.c_int64),
    ]


class _Problem(ctypes.Structure):
    device = None  # GPU of the tensors: make_* knows it (None, of a struct filled by hand: the current one)


class tsenor_quantize_problem(_Problem):
    _fields_ = [
        ("x", ctypes.c_void_p),
        ("dtype", ctypes.c_int32),
        ("square", ctypes.c_int32),
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("ld", ctypes.c_int64),
        ("mask", ctypes.c_void_p),
        ("out", tsenor_scaled),
        ("out_t", tsenor_scaled),
    ]


class tsenor_norm_problem(_Problem):
    _fields_ = [
        ("x", ctypes.c_void_p),
        ("residual", ctypes.c_void_p),
        ("gain", ctypes.c_void_p),
        ("dtype", ctypes.c_int32),
        ("gain_dtype", ctypes.c_int32),
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("ld", ctypes.c_int64),
        ("residual_ld", ctypes.c_int64),
        ("eps", ctypes.c_double),
        ("sum_out", ctypes.c_void_p),
        ("y_out", ctypes.c_void_p),
        ("out", tsenor_scaled),
    ]


class tsenor_norm_backward_problem(_Problem):
    _fields_ = [
        ("h", ctypes.c_void_p),
        ("gain", ctypes.c_void_p),
        ("dy", ctypes.c_void_p),
        ("dsum", ctypes.c_void_p),
        ("dtype", ctypes.c_int32),
        ("gain_dtype", ctypes.c_int32),
        ("rows", ctypes.c_int64),
        ("cols", ctypes.c_int64),
        ("ld", ctypes.c_int64),
        ("dy_ld", ctypes.c_int64),
        ("dsum_ld", ctypes.c_int64),
        ("eps", ctypes.c_double),
        ("dh_out", ctypes.c_void_p),
        ("dgain_out", ctypes.c_void_p),
    ]


class tsenor_product_problem(_Problem):
    _fields_ = [
        ("a", tsenor_scaled),
        ("b", tsenor_scaled),
        ("out", ctypes.c_void_p),
        ("out_ld", ctypes.c_int64),
        ("mask", ctypes.c_void_p),
    ]


class tsenor_gradient(ctypes.Structure):
    _fields_ = [
        ("in_", ctypes.c_void_p),  # `in` in C
        ("out", ctypes.c_void_p),
        ("count", ctypes.c_int64),
        ("dtype", ctypes.c_int32),
    ]


class tsenor_clip_problem(_Problem):
    _fields_ = [
        ("gradients", ctypes.POINTER(tsenor_gradient)),
        ("count", ctypes.c_int32),
        ("max_norm", ctypes.c_double),
        ("norm_out", ctypes.c_void_p),
    ]


def declare(lib) -> None:
    """Argument and result types of the entry points; called by ``binding.load``."""
    P, size, ws = ctypes.POINTER, ctypes.c_size_t, [ctypes.c_void_p, ctypes.c_size_t]
    stream = [ctypes.c_void_p]
    for name, problem, workspace in (("tsenor_quantize", tsenor_quantize_problem, False), ("tsenor_norm", tsenor_norm_problem, False),
                                     ("tsenor_norm_backward", tsenor_norm_backward_problem, True),
                                     ("tsenor_product", tsenor_product_problem, True), ("tsenor_clip", tsenor_clip_problem, True)):
        f = getattr(lib, name)
        f.argtypes, f.restype = [P(problem)] + (ws if workspace else []) + stream, ctypes.c_int
        if workspace:
            f = getattr(lib, name + "_workspace_bytes")
            f.argtypes, f.restype = [P(problem)], size


# ---- scaled matrices ----------------------------------------------------------------------------------------------------

@dataclass
class ScaledMatrix:
    """rows x cols in 8-bit floating point: ``values`` (rows, ld) float8_e4m3fn, zeros from cols to the next multiple of 128;
    ``scales`` (ceil(cols / 128), scale_ld) float8_e8m0fnu, one power of two for each column block and row."""
    values: Any
    scales: Any
    rows: int
    cols: int

    def struct(self) -> tsenor_scaled:
        # (the stride of a dimension of one row or block is whatever torch made of it)
        ld = self.values.stride(0) if self.rows > 1 else _round_up(max(self.cols, 1), TSENOR_SCALE_BLOCK)
        scale_ld = self.scales.stride(0) if self.cols > TSENOR_SCALE_BLOCK else _round_up(max(self.rows, 1), 16)
        return tsenor_scaled(self.values.data_ptr(), self.scales.data_ptr(), self.rows, self.cols, ld, scale_ld)

    def dequantize(self):
        """The values that the matrix stands for, float32 (a convenience of torch operations, for checks)."""
        import torch

        scales = self.scales[:, :self.rows].view(torch.float8_e8m0fnu).float().t()
        return self.values[:, :self.cols].float() * scales.repeat_interleave(TSENOR_SCALE_BLOCK, 1)[:, :self.cols]


def _round_up(n: int, to: int) -> int:
    return -(-n // to) * to


def empty_scaled(rows: int, cols: int, device) -> ScaledMatrix:
    """Memory for a scaled matrix, to be filled by ``tsenor_quantize`` or ``tsenor_norm``."""
    import torch

    blocks = _round_up(cols, TSENOR_SCALE_BLOCK) // TSENOR_SCALE_BLOCK
    # (at least one row and block, so that a matrix without elements has an address too)
    values = torch.empty((max(rows, 1), max(blocks, 1) * TSENOR_SCALE_BLOCK), dtype=torch.float8_e4m3fn, device=device)
    scales = torch.empty((max(blocks, 1), max(_round_up(rows, 16), 16)), dtype=torch.uint8, device=device)
    return ScaledMatrix(values[:rows], scales.view(torch.float8_e8m0fnu)[:blocks], rows, cols)


def scaled_matrix(values, scales, cols: int) -> ScaledMatrix:
    """A scaled matrix of tensors that a program already has (see ScaledMatrix for what they hold)."""
    import torch

    if values.dtype != torch.float8_e4m3fn or scales.dtype not in (torch.float8_e8m0fnu, torch.uint8):
        raise TypeError(f"values must be float8_e4m3fn and scales float8_e8m0fnu or uint8, got {values.dtype} and {scales.dtype}")
    if values.device != scales.device:
        raise ValueError("values and scales must be on one device")
    if values.dim() != 2 or scales.dim() != 2 or values.stride(1) != 1 or scales.stride(1) != 1:
        raise ValueError("values and scales must be 2-D tensors with unit column stride")
    if values.shape[1] < _round_up(cols, TSENOR_SCALE_BLOCK):
        raise ValueError("a row of values must reach to the multiple of 128 that holds its last column")
    if scales.shape[0] < -(-cols // TSENOR_SCALE_BLOCK) or scales.shape[1] < values.shape[0]:
        raise ValueError("scales must be (ceil(cols / 128), rows or more)")
    blocks, rows = -(-cols // TSENOR_SCALE_BLOCK), values.shape[0]
    reach = scales.storage_offset() + max(blocks - 1, 0) * scales.stride(0) + _round_up(rows, 16)
    if blocks and reach > scales.untyped_storage().nbytes():
        raise ValueError("each block of scales must reach to the multiple of 16 that holds the last row")
    return ScaledMatrix(values, scales, values.shape[0], cols)


# ---- describing calls ---------------------------------------------------------------------------------------------------

def _code(t, name: str) -> int:
    import torch

    if t.dtype == torch.float32:
        return TSENOR_F32
    if t.dtype == torch.bfloat16:
        return TSENOR_BF16
    raise TypeError(f"{name} must be float32 or bfloat16, got {t.dtype}")


def _matrix(t, name: str, like=None) -> None:
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{name} must be a 2-D tensor with unit column stride")
    if t.shape[0] > 1 and t.stride(0) < t.shape[1]:
        raise ValueError(f"rows of {name} must not overlap")
    if like is not None and (t.dtype != like.dtype or t.shape != like.shape):
        raise ValueError(f"{name} must have the shape and dtype of the matrix it goes with")


def _ld(t) -> int:
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]  # (the stride of a single row is whatever torch made of it)


def _whole(t, name: str, like) -> None:
    _matrix(t, name, like)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _scaled(q, name: str, rows: int, cols: int) -> None:
    # (one without elements would have no address, which stands for "not wanted")
    if q is not None and (q.rows, q.cols) != (rows, cols):
        raise ValueError(f"{name} must be a scaled matrix of {rows} x {cols}")


def _mask(mask, shape) -> None:
    import torch

    if mask.dtype not in (torch.uint8, torch.bool) or mask.shape != shape or not mask.is_contiguous():
        raise ValueError("mask must be a contiguous uint8 or bool matrix of the shape it applies to")


def _one_device(**tensors) -> int:
    where = {name: t.device for name, t in tensors.items() if t is not None}
    if any(d.type != "cuda" for d in where.values()) or len(set(where.values())) > 1:
        raise ValueError(f"all tensors must be on one GPU, got {where}")
    return next(iter(where.values())).index


def make_quantize(x, *, out: ScaledMatrix | None = None, out_t: ScaledMatrix | None = None, mask=None,
                  square: bool = False) -> tsenor_quantize_problem:
    """x (rows, cols) into ``out`` (rows, cols) and its transpose into ``out_t`` (cols, rows)."""
    _matrix(x, "x")
    if mask is not None:
        _mask(mask, x.shape)
    _scaled(out, "out", x.shape[0], x.shape[1])
    _scaled(out_t, "out_t", x.shape[1], x.shape[0])
    device = _one_device(x=x, mask=mask, out=out and out.values, out_t=out_t and out_t.values)
    p = tsenor_quantize_problem(x=x.data_ptr(), dtype=_code(x, "x"), square=int(square), rows=x.shape[0], cols=x.shape[1], ld=_ld(x),
                                mask=None if mask is None else mask.data_ptr())
    if out is not None:
        p.out = out.struct()
    if out_t is not None:
        p.out_t = out_t.struct()
    p.device = device
    return p


def make_norm(x, gain, eps: float, *, residual=None, out: ScaledMatrix | None = None, sum_out=None, y_out=None) -> tsenor_norm_problem:
    """h = x + residual into ``sum_out``; its norm times ``gain`` into ``out`` (8 bits) and ``y_out``."""
    _matrix(x, "x")
    if gain.shape != (x.shape[1],) or not gain.is_contiguous():
        raise ValueError("gain must be a contiguous vector with an element for each column")
    if residual is not None:
        _matrix(residual, "residual", x)
    for t, name in ((sum_out, "sum_out"), (y_out, "y_out")):
        if t is not None:
            _whole(t, name, x)
    _scaled(out, "out", x.shape[0], x.shape[1])
    device = _one_device(x=x, gain=gain, residual=residual, sum_out=sum_out, y_out=y_out, out=out and out.values)
    p = tsenor_norm_problem(x=x.data_ptr(), gain=gain.data_ptr(), dtype=_code(x, "x"), gain_dtype=_code(gain, "gain"),
                            rows=x.shape[0], cols=x.shape[1], ld=_ld(x), eps=float(eps))
    if residual is not None:
        p.residual, p.residual_ld = residual.data_ptr(), _ld(residual)
    p.sum_out = None if sum_out is None else sum_out.data_ptr()
    p.y_out = None if y_out is None else y_out.data_ptr()
    if out is not None:
        p.out = out.struct()
    p.device = device
    return p


def make_norm_backward(h, gain, eps: float, dy, *, dh, dgain, dsum=None) -> tsenor_norm_backward_problem:
    """dL/dh into ``dh`` and dL/dgain (float32) into ``dgain``, from h as the norm saw it, dL/dy and the gradient ``dsum`` that
    reaches h past the norm."""
    import torch

    _matrix(h, "h")
    if gain.shape != (h.shape[1],) or not gain.is_contiguous():
        raise ValueError("gain must be a contiguous vector with an element for each column")
    if dgain.dtype != torch.float32 or dgain.shape != (h.shape[1],) or not dgain.is_contiguous():
        raise ValueError("dgain must be a contiguous float32 vector with an element for each column")
    _matrix(dy, "dy", h)
    _whole(dh, "dh", h)
    if dsum is not None:
        _matrix(dsum, "dsum", h)
    device = _one_device(h=h, gain=gain, dy=dy, dh=dh, dgain=dgain, dsum=dsum)
    p = tsenor_norm_backward_problem(h=h.data_ptr(), gain=gain.data_ptr(), dy=dy.data_ptr(), dtype=_code(h, "h"),
                                     gain_dtype=_code(gain, "gain"), rows=h.shape[0], cols=h.shape[1], ld=_ld(h), dy_ld=_ld(dy),
                                     eps=float(eps), dh_out=dh.data_ptr(), dgain_out=dgain.data_ptr())
    if dsum is not None:
        p.dsum, p.dsum_ld = dsum.data_ptr(), _ld(dsum)
    p.device = device
    return p


def make_product(a: ScaledMatrix, b: ScaledMatrix, *, out, mask=None) -> tsenor_product_problem:
    """a b^T into ``out`` (a.rows, b.rows), bfloat16."""
    import torch

    _matrix(out, "out")
    if out.dtype != torch.bfloat16 or out.shape != (a.rows, b.rows):
        raise ValueError("out must be a bfloat16 matrix of a.rows x b.rows")
    if a.cols != b.cols:
        raise ValueError("a and b must have the same number of columns")
    if mask is not None:
        _mask(mask, out.shape)
    device = _one_device(a=a.values, a_scales=a.scales, b=b.values, b_scales=b.scales, out=out, mask=mask)
    p = tsenor_product_problem(a=a.struct(), b=b.struct(), out=out.data_ptr(), out_ld=_ld(out),
                               mask=None if mask is None else mask.data_ptr())
    p.device = device
    return p


def make_clip(gradients, max_norm: float, *, norm_out, out=None) -> tsenor_clip_problem:
    """The gradients scaled down to ``max_norm`` into ``out`` (None: in place), norm and factor into ``norm_out``."""
    import torch

    gradients = list(gradients)
    out = gradients if out is None else list(out)
    if len(out) != len(gradients):
        raise ValueError("out must have a tensor for each gradient")
    if norm_out.dtype != torch.float32 or norm_out.numel() != 2 or not norm_out.is_contiguous():
        raise ValueError("norm_out must be a contiguous float32 tensor of 2 elements")
    table = (tsenor_gradient * max(len(gradients), 1))()
    for k, (g, o) in enumerate(zip(gradients, out)):
        if not g.is_contiguous() or not o.is_contiguous() or o.dtype != g.dtype or o.numel() != g.numel():
            raise ValueError("gradients and out must be contiguous, with the same elements and dtypes")
        _one_device(gradient=g, out=o, norm_out=norm_out)
        table[k] = tsenor_gradient(g.data_ptr(), o.data_ptr(), g.numel(), _code(g, "gradient"))
    p = tsenor_clip_problem(gradients=table, count=len(gradients), max_norm=float(max_norm), norm_out=norm_out.data_ptr())
    p.device = _one_device(norm_out=norm_out)
    return p


# ---- the calls ------------------------------------------------------------------------------------------------------------

def _enqueue(name: str, problem, stream, *scratch) -> None:
    here = current_device()
    device = here if problem.device is None else problem.device
    if device != here:  # a launch goes to the current GPU
        import torch

        with torch.cuda.device(device):
            _enqueue(name, problem, stream, *scratch)
        return
    rc = getattr(load(), name)(ctypes.byref(problem), *scratch, current_stream(device) if stream is None else stream.cuda_stream)
    if rc != TSENOR_OK:
        raise TsenorError(rc, name)


def _scratch(workspace, problem):
    if workspace is None:
        return None, 0
    if not workspace.is_contiguous() or workspace.get_device() != (current_device() if problem.device is None else problem.device):
        raise ValueError("workspace must be contiguous and on the GPU of the tensors")
    return ctypes.c_void_p(workspace.data_ptr()), workspace.numel() * workspace.element_size()


def tsenor_quantize(problem: tsenor_quantize_problem, stream=None) -> None:
    _enqueue("tsenor_quantize", problem, stream)


def tsenor_norm(problem: tsenor_norm_problem, stream=None) -> None:
    _enqueue("tsenor_norm", problem, stream)


def tsenor_norm_backward_workspace_bytes(problem: tsenor_norm_backward_problem) -> int:
    return int(load().tsenor_norm_backward_workspace_bytes(ctypes.byref(problem)))


def tsenor_norm_backward(problem: tsenor_norm_backward_problem, workspace=None, stream=None) -> None:
    _enqueue("tsenor_norm_backward", problem, stream, *_scratch(workspace, problem))


def tsenor_product_workspace_bytes(problem: tsenor_product_problem) -> int:
    return int(load().tsenor_product_workspace_bytes(ctypes.byref(problem)))


def tsenor_product(problem: tsenor_product_problem, workspace=None, stream=None) -> None:
    _enqueue("tsenor_product", problem, stream, *_scratch(workspace, problem))


def tsenor_clip_workspace_bytes(problem: tsenor_clip_problem) -> int:
    return int(load().tsenor_clip_workspace_bytes(ctypes.byref(problem)))


def tsenor_clip(problem: tsenor_clip_problem, workspace, stream=None) -> None:
    _enqueue("tsenor_clip", problem, stream, *_scratch(workspace, problem))
