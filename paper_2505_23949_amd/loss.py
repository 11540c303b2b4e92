"""ctypes binding of the losses of libtsenor.so (declared in include/tsenor_loss.h): softmax cross entropy over a vocabulary and
distillation from a teacher's top logits, both from hidden states through the product with the head, with their gradients.

As in ``layer``: ``make_*`` describes a call once (no copies; the tensors must outlive it), the function named like the C entry point
enqueues it as often as wanted, on the current stream of the GPU that the tensors are on (on ``stream`` if given).
"""
from __future__ import annotations

import ctypes

from .binding import load
from .layer import _code, _enqueue, _ld, _matrix, _one_device, _Problem, _scratch, _whole

TSENOR_LOSS_MAX_ENTRIES = 256


class tsenor_head(ctypes.Structure):
    _fields_ = [
        ("h", ctypes.c_void_p),
        ("weight", ctypes.c_void_p),
        ("dtype", ctypes.c_int32),
        ("tokens", ctypes.c_int64),
        ("vocab", ctypes.c_int64),
        ("width", ctypes.c_int64),
        ("h_ld", ctypes.c_int64),
        ("weight_ld", ctypes.c_int64),
        ("dloss", ctypes.c_void_p),
        ("loss_out", ctypes.c_void_p),
        ("lse_out", ctypes.c_void_p),
        ("dh_out", ctypes.c_void_p),
        ("dweight_out", ctypes.c_void_p),
    ]


class tsenor_cross_entropy_problem(_Problem):
    _fields_ = [
        ("head", tsenor_head),
        ("targets", ctypes.c_void_p),
    ]


class tsenor_distill_problem(_Problem):
    _fields_ = [
        ("head", tsenor_head),
        ("ids", ctypes.c_void_p),
        ("logits", ctypes.c_void_p),
        ("logits_dtype", ctypes.c_int32),
        ("k", ctypes.c_int32),
        ("ids_ld", ctypes.c_int64),
        ("logits_ld", ctypes.c_int64),
        ("temperature", ctypes.c_double),
    ]


def declare(lib) -> None:
    """Argument and result types of the entry points; called by ``binding.load``."""
    for name, problem in (("tsenor_cross_entropy", tsenor_cross_entropy_problem), ("tsenor_distill", tsenor_distill_problem)):
        f = getattr(lib, name)
        f.argtypes, f.restype = [ctypes.POINTER(problem), ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p], ctypes.c_int
        f = getattr(lib, name + "_workspace_bytes")
        f.argtypes, f.restype = [ctypes.POINTER(problem)], ctypes.c_size_t


# ---- describing calls ---------------------------------------------------------------------------------------------------

def _floats(t, name: str, tokens: int):
    import torch

    if t is None:
        return None
    if t.dtype != torch.float32 or t.shape != (tokens,) or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous float32 vector with an element for each token")
    return t.data_ptr()


def _head(h, weight, dloss, loss, lse, dh, dweight) -> tsenor_head:
    _matrix(h, "h")
    _matrix(weight, "weight")
    if weight.dtype != h.dtype or weight.shape[1] != h.shape[1]:
        raise ValueError("weight must have the dtype of h and as many columns")
    for t, name, like in ((dh, "dh", h), (dweight, "dweight", weight)):
        if t is not None:
            _whole(t, name, like)
    tokens = h.shape[0]
    p = tsenor_head(h=h.data_ptr(), weight=weight.data_ptr(), dtype=_code(h, "h"), tokens=tokens, vocab=weight.shape[0], width=h.shape[1],
                    h_ld=_ld(h), weight_ld=_ld(weight), dloss=_floats(dloss, "dloss", tokens), loss_out=_floats(loss, "loss", tokens),
                    lse_out=_floats(lse, "lse", tokens))
    # (a matrix without elements has no address, which is the same as one that is not wanted)
    p.dh_out = None if dh is None else dh.data_ptr()
    p.dweight_out = None if dweight is None else dweight.data_ptr()
    return p


def make_cross_entropy(h, weight, targets, *, loss, lse=None, dloss=None, dh=None, dweight=None) -> tsenor_cross_entropy_problem:
    """The cross entropy of each token into ``loss`` (float32), from hidden states h (tokens, width), the head ``weight`` (vocab, width)
    and int64 ``targets`` (tokens), one outside the vocabulary (such as -100) leaving its token out.  The logarithm of the sum of
    exponentials into ``lse``; the gradients of sum(dloss * loss) into ``dh`` and ``dweight`` (``dloss`` None: of the sum)."""
    import torch

    if targets.dtype != torch.int64 or targets.shape != (h.shape[0],) or not targets.is_contiguous():
        raise ValueError("targets must be a contiguous int64 vector with an element for each token")
    device = _one_device(h=h, weight=weight, targets=targets, loss=loss, lse=lse, dloss=dloss, dh=dh, dweight=dweight)
    p = tsenor_cross_entropy_problem(head=_head(h, weight, dloss, loss, lse, dh, dweight), targets=targets.data_ptr())
    p.device = device
    return p


def make_distill(h, weight, ids, logits, *, loss, temperature: float = 1.0, lse=None, dloss=None, dh=None,
                 dweight=None) -> tsenor_distill_problem:
    """The divergence of each token's distribution from its teacher's into ``loss`` (float32): int64 ``ids`` and ``logits`` (float32 or
    bfloat16), both (tokens, k), are the teacher's top words, and entries whose id is outside the vocabulary take no part.  Both
    sides' logits are divided by ``temperature``.  Otherwise as ``make_cross_entropy``."""
    import torch

    _matrix(ids, "ids")
    _matrix(logits, "logits")
    if ids.dtype != torch.int64 or ids.shape[0] != h.shape[0] or logits.shape != ids.shape:
        raise ValueError("ids must be an int64 matrix with a row for each token, and logits a matrix of its shape")
    device = _one_device(h=h, weight=weight, ids=ids, logits=logits, loss=loss, lse=lse, dloss=dloss, dh=dh, dweight=dweight)
    p = tsenor_distill_problem(head=_head(h, weight, dloss, loss, lse, dh, dweight), ids=ids.data_ptr(), logits=logits.data_ptr(),
                               logits_dtype=_code(logits, "logits"), k=ids.shape[1], ids_ld=_ld(ids), logits_ld=_ld(logits),
                               temperature=float(temperature))
    p.device = device
    return p


# ---- the calls ------------------------------------------------------------------------------------------------------------

def tsenor_cross_entropy_workspace_bytes(problem: tsenor_cross_entropy_problem) -> int:
    return int(load().tsenor_cross_entropy_workspace_bytes(ctypes.byref(problem)))


def tsenor_cross_entropy(problem: tsenor_cross_entropy_problem, workspace, stream=None) -> None:
    _enqueue("tsenor_cross_entropy", problem, stream, *_scratch(workspace, problem))


def tsenor_distill_workspace_bytes(problem: tsenor_distill_problem) -> int:
    return int(load().tsenor_distill_workspace_bytes(ctypes.byref(problem)))


def tsenor_distill(problem: tsenor_distill_problem, workspace, stream=None) -> None:
    _enqueue("tsenor_distill", problem, stream, *_scratch(workspace, problem))
