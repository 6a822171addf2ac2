"""The distillation loss of a student's logits against a teacher's k best, under the token mask, for torch's training loops.

The teacher's lists are what `Pre3.apply_mask_topk` writes; definitions are beside pre3_distill_loss in include/pre3.h.  Everything runs
on the current stream; results, gradients and workspaces are allocated by torch.
"""
from __future__ import annotations

import ctypes

import torch

from . import binding as B

B.load()


def _arguments(logits, teacher_ids, teacher_logits, bitmask, temperature):
    """The call's arguments as the library takes them, and the workspace, which has to live until the call returns.  What does
    not fit raises here.  (A small call's kernels take some 6 us: nothing is asked of torch twice.)"""
    shape, ids_shape = logits.shape, teacher_ids.shape
    assert len(shape) == 2 and len(ids_shape) == 2
    (rows, vocab), (stride, one) = shape, logits.stride()
    assert (one == 1 or vocab == 1) and ids_shape[0] == rows and teacher_logits.shape == ids_shape
    assert teacher_ids.is_contiguous() and teacher_logits.is_contiguous()
    device = logits.device
    assert teacher_ids.device == device and teacher_logits.device == device, "tensors on several devices"
    mask = None
    if bitmask is not None:
        assert bitmask.shape == (rows, (vocab + 31) // 32) and bitmask.is_contiguous() and bitmask.device == device
        mask = B._dev(bitmask, "u32")
    if rows <= 1:
        stride = max(stride, vocab)                     # (the stride of a single row may be anything)
    d = B._Distill(B._dev(logits, "logits"), mask, B._dev(teacher_ids, "i32"), B._dev(teacher_logits, "logits"), stride,
                   B._LOGITS_TYPE[logits.dtype], B._LOGITS_TYPE[teacher_logits.dtype], rows, vocab, ids_shape[1], temperature, None, 0)
    workspace = None
    need = B._lib.pre3_distill_workspace_bytes(rows, vocab)
    if need > 0:
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        d.workspace, d.workspace_bytes = workspace.data_ptr(), need
    return d, workspace


def _call(name, device, *arguments):
    """The library launches on the current device, so the tensors' one has to be that."""
    if B._current_device() == device.index:
        rc = getattr(B._lib, name)(*arguments, B._stream_ptr(None))
    else:
        with torch.cuda.device(device):
            rc = getattr(B._lib, name)(*arguments, B._stream_ptr(None))
    if rc != B.PRE3_OK:
        raise B.Pre3Error(rc, f"{name}: bad argument or launch failure")


class _DistillLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, teacher_ids, teacher_logits, bitmask, temperature):
        d, workspace = _arguments(logits, teacher_ids, teacher_logits, bitmask, temperature)
        device, rows = logits.device, d.rows
        loss = torch.empty(rows, dtype=torch.float32, device=device)
        if not ctx.needs_input_grad[0]:
            _call("pre3_distill_loss", device, ctypes.byref(d), loss.data_ptr(), None)
        else:
            stats = torch.empty(2 * rows, dtype=torch.float32, device=device)
            _call("pre3_distill_loss", device, ctypes.byref(d), loss.data_ptr(), stats.data_ptr())
            ctx.save_for_backward(logits, teacher_ids, teacher_logits, bitmask, stats)
            ctx.arguments = d
        return loss

    @staticmethod
    def backward(ctx, weight):
        if torch.is_grad_enabled():                     # create_graph=True
            raise RuntimeError("distill_loss is differentiable once")
        logits, _, _, _, stats = ctx.saved_tensors      # (raises where one of them has been written since)
        d = ctx.arguments
        grad = torch.empty((d.rows, d.vocab), dtype=logits.dtype, device=logits.device)
        _call("pre3_distill_grad", logits.device, ctypes.byref(d), stats.data_ptr(), B._dev(weight, "f32"), weight.stride(0), grad.data_ptr(), d.vocab)
        return grad, None, None, None, None


def distill_loss(logits, teacher_ids, teacher_logits, bitmask=None, temperature: float = 1.0):
    """The loss [rows] (float32) of `logits` [rows, vocab] (bfloat16, float16 or float32, rows may be strided) against the teacher's lists
    `teacher_ids` (int32, -1 padded) and `teacher_logits` [rows, k], k <= 256; `bitmask` [rows, ceil(vocab / 32)] or None.  Differentiable
    once, with respect to `logits`: the backward pass reads them again, so they may not be overwritten before."""
    return _DistillLoss.apply(logits, teacher_ids, teacher_logits, bitmask, float(temperature))


def distill_loss_grad(logits, teacher_ids, teacher_logits, bitmask=None, temperature: float = 1.0, row_weight=None, out=None):
    """(loss, gradient) at once: the losses of `distill_loss` and the gradient of their sum, each times its `row_weight` [rows] (float32;
    None: 1).  The gradient has the type of `logits` and goes to `out` if given, which may be `logits` itself.  For a training step that
    hands the gradient on by itself, `x.backward(gradient)`: the logits come from memory once, where `distill_loss` and its backward
    pass fetch them twice."""
    logits = logits.detach()
    d, workspace = _arguments(logits, teacher_ids, teacher_logits, bitmask, float(temperature))
    device, rows, vocab = logits.device, d.rows, d.vocab
    if out is None:
        out = torch.empty((rows, vocab), dtype=logits.dtype, device=device)
    assert out.shape == (rows, vocab) and out.dtype == logits.dtype and (out.stride(1) == 1 or vocab == 1) and out.device == device
    weight, weight_stride = None, 0
    if row_weight is not None:
        assert row_weight.shape == (rows,) and row_weight.device == device
        weight, weight_stride = B._dev(row_weight, "f32"), row_weight.stride(0)
    loss = torch.empty(rows, dtype=torch.float32, device=device)
    _call("pre3_distill_loss_grad", device, ctypes.byref(d), weight, weight_stride, loss.data_ptr(), out.data_ptr(),
          out.stride(0) if rows > 1 else max(out.stride(0), vocab))
    return loss, out
