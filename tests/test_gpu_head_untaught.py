"""Batches of which no row teaches (a prompt's tokens, padding), where the gradient of the weights is summed in shares along the rows: zeros, whatever the workspace
held before."""
import ctypes as c

import pytest
import torch

from test_gpu_head_loss import TYPES, inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,vocab,dim", [("bf16", 4346, 143, 154), ("bf16", 8192, 8000, 64), ("f16", 4000, 140001, 64), ("f32", 2000, 400, 24)])
@pytest.mark.parametrize("masked", [False, True])
def test_no_row_teaches(dtype, rows, vocab, dim, masked):
    from torch.profiler import ProfilerActivity, profile
    from test_matrices_arguments import Head, lib
    print(f"[head] {dtype} {rows} x {vocab} x {dim} masked {masked}", flush=True)
    hidden, weight, targets, _, g = inputs(dtype, rows, vocab, dim, None, seed=31)
    bits = torch.zeros((rows, -(-vocab // 32)), dtype=torch.int32, device="cuda") if masked else None
    targets = targets.clamp(0, vocab - 1) if masked else torch.full_like(targets, -1)
    head = Head(hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), bits.data_ptr() if masked else None, dim, dim, list(TYPES).index(dtype), 4, rows, vocab, dim)
    need = max(lib().pre3_head_workspace_bytes(c.byref(head), grads) for grads in (0, 1))
    workspace = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    head.workspace, head.workspace_bytes = (workspace.data_ptr() + 255) // 256 * 256, need
    stream = torch.cuda.current_stream().cuda_stream

    def out():
        workspace.fill_(255)                                        # (NaNs, in every type)
        return torch.full((rows,), 9.0, device="cuda"), torch.full_like(hidden, 9.0), torch.full_like(weight, 9.0)

    loss, d_h, d_w = out()
    with profile(activities=[ProfilerActivity.CUDA]) as prof:
        assert lib().pre3_head_loss_grad(c.byref(head), g.data_ptr(), 1, loss.data_ptr(), d_h.data_ptr(), dim, d_w.data_ptr(), dim, stream) == 0
        torch.cuda.synchronize()
    assert "head_weight_grad_kernel" not in " ".join(e.key for e in prof.key_averages())      # (that sums all rows in one share)
    assert not loss.any() and not d_h.any() and not d_w.any()

    loss, d_h, d_w = out()
    stats = torch.empty((rows, 2), device="cuda")
    assert lib().pre3_head_loss(c.byref(head), loss.data_ptr(), stats.data_ptr(), stream) == 0
    workspace.fill_(255)
    assert lib().pre3_head_grad(c.byref(head), stats.data_ptr(), g.data_ptr(), 1, d_h.data_ptr(), dim, d_w.data_ptr(), dim, stream) == 0
    assert not loss.any() and not d_h.any() and not d_w.any()
