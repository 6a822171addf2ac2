"""Loss and gradients of heads whose vocabulary is worked on in several pieces (what one takes of the workspace is held below a gigabyte), against the definition
in 64 bits, within the bounds that test_gpu_head_loss derives."""
import ctypes as c

import pytest
import torch

from test_gpu_head_loss import TYPES, close, inputs, pack, reference

pytestmark = pytest.mark.gpu


def pieces_of(call):
    """A call's results, and the pieces that it has made slopes of."""
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as prof:
        got = call()
        torch.cuda.synchronize()
    return got, sum(e.count for e in prof.key_averages() if "head_row_slopes_kernel" in e.key or "head_slopes_kernel" in e.key)


def whole(dtype, rows, vocab, dim, strided=False):
    print(f"[head] {dtype} {rows} x {vocab} x {dim} strided {strided}", flush=True)
    hidden, weight, targets, allowed, g = inputs(dtype, rows, vocab, dim, "mixed", seed=rows + dim, strided=strided)
    targets[rows - 1] = vocab - 1                                  # a target of the last piece
    allowed[rows - 1, vocab - 1] = True
    if dtype == "f16":
        g = g * 2.0 ** 10                                          # (a token's share of so many is small: gradients of normal numbers)
    return hidden, weight, targets, allowed, g, pack(allowed), reference(hidden, weight, targets, allowed, g, dtype)


# Few rows, whose logits are kept as long as the call, or from the loss's to the gradients'.
@pytest.mark.parametrize("dtype,rows,vocab,dim,strided,pieces", [("f32", 40, 360001, 1000, False, 3), ("f32", 9, 200001, 1000, True, 2), ("bf16", 40, 500001, 1001, False, 2),
                                                                 ("f16", 5, 500001, 1001, True, 2)])
def test_few_rows(dtype, rows, vocab, dim, strided, pieces):
    from paper_2506_03887_amd import head_loss, head_loss_grad
    from test_matrices_arguments import Head, lib
    hidden, weight, targets, allowed, g, bits, want = whole(dtype, rows, vocab, dim, strided)

    def check(got):
        for x, y, what in zip(got, want, ("loss", "hidden", "weight")):
            close(x, y, what)

    got, made = pieces_of(lambda: head_loss_grad(hidden, weight, targets, bits, row_weight=g))
    assert made == pieces
    check(got)
    # (a loss's call may cut the vocabulary otherwise, and where a tile's sums begin depends on its place in a piece: other last bits within the same bounds)
    h, w = hidden.detach().requires_grad_(), weight.detach().requires_grad_()
    loss = head_loss(h, w, targets, bits)
    check((loss.detach(), *torch.autograd.grad(loss, (h, w), g)))  # of the logits that the loss's call has kept
    del loss, h, w
    # the gradients' call makes the logits again
    head = Head(hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), bits.data_ptr(), hidden.stride(0), weight.stride(0), list(TYPES).index(dtype), 4, rows, vocab, dim)
    need = max(lib().pre3_head_workspace_bytes(c.byref(head), grads) for grads in (0, 1))
    workspace = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    head.workspace, head.workspace_bytes = (workspace.data_ptr() + 255) // 256 * 256, need
    loss, stats = torch.empty(rows, device="cuda"), torch.empty((rows, 2), device="cuda")
    d_h, d_w = torch.empty_like(got[1]), torch.empty_like(got[2])
    stream = torch.cuda.current_stream().cuda_stream
    assert lib().pre3_head_loss(c.byref(head), loss.data_ptr(), stats.data_ptr(), stream) == 0
    assert lib().pre3_head_grad(c.byref(head), stats.data_ptr(), g.data_ptr(), 1, d_h.data_ptr(), dim, d_w.data_ptr(), dim, stream) == 0
    check((loss, d_h, d_w))


# Rows whose logits are made again for the gradients, tile by tile: packed weights, and weights as they lie.
@pytest.mark.parametrize("dtype,rows,vocab,dim,strided,pieces", [("f32", 300, 340001, 520, False, 3), ("f16", 2000, 180001, 1001, True, 2), ("bf16", 4000, 140001, 64, False, 2)])
def test_many_rows(dtype, rows, vocab, dim, strided, pieces):
    from paper_2506_03887_amd import head_loss, head_loss_grad
    hidden, weight, targets, allowed, g, bits, want = whole(dtype, rows, vocab, dim, strided)
    got, made = pieces_of(lambda: head_loss_grad(hidden, weight, targets, bits, row_weight=g))
    assert made == pieces
    h, w = hidden.detach().requires_grad_(), weight.detach().requires_grad_()
    loss = head_loss(h, w, targets, bits)
    by_autograd, made = pieces_of(lambda: torch.autograd.grad(loss, (h, w), g, retain_graph=True))
    assert made == pieces
    h_only, = torch.autograd.grad(loss, (h,), g, retain_graph=True)
    w_only, = torch.autograd.grad(loss, (w,), g)
    for results in (got, (loss.detach(), *by_autograd), (loss.detach(), h_only, w_only)):
        for x, y, what in zip(results, want, ("loss", "hidden", "weight")):
            close(x, y, what)
