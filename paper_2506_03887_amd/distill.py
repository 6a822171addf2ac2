"""The distillation loss of a student's logits against a teacher's k best, under the token mask, for torch's training loops.

The teacher's lists are what `Pre3.apply_mask_topk` writes; definitions are beside pre3_distill_loss in include/pre3.h.  Everything runs
on the current stream; results, gradients and workspaces are allocated by torch.  What checks the tensors and stands in the autograd
graph is csrc/torch_distill.cpp.
"""
from __future__ import annotations

import os

from . import binding as B

B.load()
if not os.path.exists(os.path.join(os.path.dirname(__file__), "_torch_distill.so")):
    raise ImportError("_torch_distill.so is missing: build it with paper_2506_03887_amd.build.build_torch()")
from . import _torch_distill as _torch  # noqa: E402  (libpre3.so first, and before that torch and its HIP runtime)

_torch.raise_as(B.Pre3Error)


def _refuse_in_fork():
    """Raises in a process forked from one that has used the GPU: it holds that one's tensors and cannot use them."""
    if B._in_bad_fork():
        B._torch.cuda.current_device()                  # raises, and says why


def distill_loss(logits, teacher_ids, teacher_logits, bitmask=None, temperature: float = 1.0):
    """The loss [rows] (float32) of `logits` [rows, vocab] (bfloat16, float16 or float32, rows may be strided) against the teacher's lists
    `teacher_ids` (int32, -1 padded) and `teacher_logits` [rows, k], k <= 256; `bitmask` [rows, ceil(vocab / 32)] or None.  Differentiable
    once, with respect to `logits`, in reverse mode.  The backward pass reads the logits, the lists and the mask again: a call of the library or an
    operation of torch that has overwritten one of them before makes it raise."""
    _refuse_in_fork()
    return _torch.distill_loss(logits, teacher_ids, teacher_logits, bitmask, float(temperature))


def distill_loss_grad(logits, teacher_ids, teacher_logits, bitmask=None, temperature: float = 1.0, row_weight=None, out=None):
    """(loss, gradient) at once: the losses of `distill_loss` and the gradient of their sum, each times its `row_weight` [rows] (float32;
    None: 1).  The gradient has the type of `logits` and goes to `out` if given, which may be `logits` itself where no other operation
    has saved them for its backward pass (autograd raises there if one has).  For a training step that hands the gradient on by itself,
    `x.backward(gradient)`: a row is read again right after its sums are there, mostly out of the caches, where the backward pass of
    `distill_loss` fetches it from memory a second time."""
    _refuse_in_fork()
    return _torch.distill_loss_grad(logits, teacher_ids, teacher_logits, bitmask, float(temperature), row_weight, out)
