"""The model's two matrices of the vocabulary's size, for torch: the table that tokens are looked up in, and the head whose product with the
hidden states gives the logits that mask, sampler and losses work on.

Definitions are beside pre3_embed, pre3_head_loss and pre3_head8_logits in include/pre3.h.  Everything runs on the current stream; results,
gradients and workspaces are allocated by torch.  A backward pass that is captured into a graph wants no eager
autograd graph of the same leaves alive, as with torch's own operations.  What checks the tensors and stands in the autograd graph is csrc/torch_matrices.cpp.
"""
from __future__ import annotations

import os

from . import binding as B

B.load()
if not os.path.exists(os.path.join(os.path.dirname(__file__), "_torch_matrices.so")):
    raise ImportError("_torch_matrices.so is missing: build it with paper_2506_03887_amd.build.build_torch()")
from . import _torch_matrices as _torch  # noqa: E402  (libpre3.so first, and before that torch and its HIP runtime)

_torch.raise_as(B.Pre3Error)


def _refuse_in_fork():
    """Raises in a process forked from one that has used the GPU: it holds that one's tensors and cannot use them."""
    if B._in_bad_fork():
        B._torch.cuda.current_device()                  # raises, and says why


def embed(weight, tokens, scale: float = 1.0, out=None):
    """Rows of `weight` [vocab, dim] (bfloat16, float16 or float32, rows may be strided) by `tokens` (int32 or int64, any shape), times `scale`:
    [*tokens' shape, dim].  An id outside 0 .. vocab - 1 (the sampler's -1, padding) gives zeros and no gradient.  Differentiable once, with
    respect to `weight`, in reverse mode; the gradient is dense, and the same inputs give the same bits.  `out`, where no gradient is asked
    for: what the rows are written to; contiguous, it may not overlap the inputs or be part of an autograd graph.  `tokens` are contiguous."""
    _refuse_in_fork()
    return _torch.embed(weight, tokens, float(scale), out)


def head_loss(hidden, weight, targets, bitmask=None):
    """The cross entropy [rows] (float32) of `targets` [rows] (int32 or int64, contiguous) in the logits `hidden` [rows, dim] @ `weight` [vocab, dim].T (both
    bfloat16, float16 or float32, rows may be strided) behind `bitmask` [rows, ceil(vocab / 32)] or None; logits are not kept but for
    the backward pass of up to 128 rows, or of more of few tokens (where a product's sums take less than 256 MiB).  A row whose target is outside 0 .. vocab - 1 or not allowed
    has loss 0 and no gradient.  Differentiable once, with respect to `hidden` and `weight`, in reverse mode; of more than
    128 rows the gradients are products of slopes rounded to the operands' type.  The backward pass reads the inputs again: a call of the library or an operation of torch that has overwritten one of
    them before makes it raise."""
    _refuse_in_fork()
    return _torch.head_loss(hidden, weight, targets, bitmask)


def head_loss_grad(hidden, weight, targets, bitmask=None, row_weight=None):
    """(loss, gradient of hidden, gradient of weight) at once: the losses of `head_loss` and the gradients of their sum, each loss times its
    `row_weight` [rows] (float32; None: 1), of the operands' type."""
    _refuse_in_fork()
    return _torch.head_loss_grad(hidden, weight, targets, bitmask, row_weight)


def quantise_rows(x):
    """(whole numbers, scale): `x` [rows, dim] (bfloat16, float16 or float32, rows may be strided) in 8 bits, int8 [rows, dim] with rows at 16-byte
    boundaries, and float32 [rows]; x is about their product.  What `head_logits` takes as a head."""
    _refuse_in_fork()
    return _torch.quantise_rows(x)


def head_logits(hidden, weight, scale, bitmask=None, out=None):
    """The logits [rows, vocab] of `hidden` [rows, dim] (bfloat16, float16 or float32, rows may be strided), which is quantised row by row on the
    way, against a head in 8 bits, `weight` [vocab, dim] and `scale` [vocab] of `quantise_rows`; -inf where `bitmask` [rows, ceil(vocab / 32)]
    has no bit.  Of the hidden states' type, in `out` if given (rows may be strided; it may not overlap the inputs or be part of an autograd graph).  For decoding: it has no gradient."""
    _refuse_in_fork()
    return _torch.head_logits(hidden, weight, scale, bitmask, out)
