"""What a head's loss holds of the GPU's memory while it runs."""
import pytest
import torch

from test_gpu_head_loss import close, inputs, pack, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,vocab,dim,most", [("f32", 16, 128256, 2048, 32), ("f16", 40, 100003, 1001, 32)])
def test_a_loss_alone_beside_a_model(dtype, rows, vocab, dim, most):
    """Few rows of weights that are read as they lie: a few MiB beside 1 GiB and 190 MiB of weights."""
    from paper_2506_03887_amd import head_loss
    print(f"[head] {dtype} {rows} x {vocab} x {dim}", flush=True)
    hidden, weight, targets, allowed, g = inputs(dtype, rows, vocab, dim, "mixed", seed=41)
    bits = pack(allowed)
    want = reference(hidden, weight, targets, allowed, g, dtype)[0]
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    loss = head_loss(hidden, weight, targets, bits)
    assert torch.cuda.max_memory_allocated() - before <= most << 20
    close(loss, want, "loss")
