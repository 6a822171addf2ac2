"""The distillation loss of a student's logits against a teacher's k best, under the token mask, for torch's training loops.

The teacher's lists are what `Pre3.apply_mask_topk` writes; definitions are beside pre3_distill_loss in include/pre3.h.  Everything runs
on the current stream; results and gradients are allocated by torch.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B


def _arguments(logits, teacher_ids, teacher_logits, bitmask, temperature):
    """The call's arguments as the library takes them; what does not fit raises here."""
    assert logits.dim() == 2 and (logits.stride(1) == 1 or logits.shape[1] == 1)
    rows, vocab = logits.shape
    assert teacher_ids.dim() == 2 and teacher_ids.shape[0] == rows and teacher_ids.is_contiguous()
    assert teacher_logits.shape == teacher_ids.shape and teacher_logits.is_contiguous()
    assert bitmask is None or (bitmask.is_contiguous() and bitmask.shape == (rows, (vocab + 31) // 32))
    devices = {t.device for t in (logits, teacher_ids, teacher_logits, bitmask) if t is not None}
    assert len(devices) == 1, "tensors on several devices"
    return B._Distill(B._dev(logits, "logits"), None if bitmask is None else B._dev(bitmask, "u32"), B._dev(teacher_ids, "i32"),
                      B._dev(teacher_logits, "logits"), _row_stride(logits), B._LOGITS_TYPE[logits.dtype],
                      B._LOGITS_TYPE[teacher_logits.dtype], rows, vocab, teacher_ids.shape[1], temperature)


def _row_stride(t):
    return t.stride(0) if t.shape[0] > 1 else max(t.stride(0), t.shape[1])      # (the stride of a single row may be anything)


def _check(rc, call):
    if rc != B.PRE3_OK:
        raise B.Pre3Error(rc, f"{call}: bad argument or launch failure")


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, teacher_ids, teacher_logits, bitmask, temperature):
        lib, rows = B.load(), logits.shape[0]
        d = _arguments(logits, teacher_ids, teacher_logits, bitmask, temperature)
        loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
        stats = torch.empty((rows, 2), dtype=torch.float32, device=logits.device) if ctx.needs_input_grad[0] else None
        with torch.cuda.device(logits.device):
            _check(lib.pre3_distill_loss(ctypes.byref(d), loss.data_ptr(), None if stats is None else stats.data_ptr(), B._stream_ptr(None)),
                   "distill_loss")
        if stats is not None:
            ctx.save_for_backward(logits, teacher_ids, teacher_logits, bitmask, stats)
            ctx.temperature = temperature
        return loss

    @staticmethod
    def backward(ctx, weight):
        if torch.is_grad_enabled():                     # create_graph=True
            raise RuntimeError("distill_loss is differentiable once")
        logits, teacher_ids, teacher_logits, bitmask, stats = ctx.saved_tensors
        d = _arguments(logits, teacher_ids, teacher_logits, bitmask, ctx.temperature)
        grad = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
        with torch.cuda.device(logits.device):
            _check(B.load().pre3_distill_grad(ctypes.byref(d), stats.data_ptr(), B._dev(weight, "f32"), weight.stride(0), grad.data_ptr(),
                                              logits.shape[1], B._stream_ptr(None)), "distill_loss, backward")
        return grad, None, None, None, None


def distill_loss(logits, teacher_ids, teacher_logits, bitmask=None, temperature: float = 1.0):
    """The loss [rows] (float32) of `logits` [rows, vocab] (bfloat16, float16 or float32, rows may be strided) against the teacher's lists
    `teacher_ids` (int32, -1 padded) and `teacher_logits` [rows, k], k <= 256; `bitmask` [rows, ceil(vocab / 32)] or None.  Differentiable
    once, with respect to `logits`: the backward pass reads them again, so they may not be overwritten before."""
    return _DistillLoss.apply(logits, teacher_ids, teacher_logits, bitmask, float(temperature))


def distill_loss_grad(logits, teacher_ids, teacher_logits, bitmask=None, temperature: float = 1.0, row_weight=None, out=None):
    """(loss, gradient) in one pass over the logits: the losses of `distill_loss` and the gradient of their sum, each times its
    `row_weight` [rows] (float32; None: 1).  The gradient has the type of `logits` and goes to `out` if given, which may be `logits`
    itself.  For a training step that hands the gradient on by itself, `x.backward(gradient)`: the logits are read and their gradient written
    once, where `distill_loss` and its backward pass read them twice."""
    lib, logits = B.load(), logits.detach()
    d = _arguments(logits, teacher_ids, teacher_logits, bitmask, float(temperature))
    rows, vocab = logits.shape
    if out is None:
        out = torch.empty((rows, vocab), dtype=logits.dtype, device=logits.device)
    assert out.shape == logits.shape and out.dtype == logits.dtype and (out.stride(1) == 1 or vocab == 1) and out.device == logits.device
    assert row_weight is None or (row_weight.shape == (rows,) and row_weight.device == logits.device)
    loss = torch.empty(rows, dtype=torch.float32, device=logits.device)
    with torch.cuda.device(logits.device):
        _check(lib.pre3_distill_loss_grad(ctypes.byref(d), None if row_weight is None else B._dev(row_weight.detach(), "f32"),
                                          0 if row_weight is None else row_weight.stride(0), loss.data_ptr(), out.data_ptr(),
                                          _row_stride(out), B._stream_ptr(None)), "distill_loss_grad")
    return loss, out
