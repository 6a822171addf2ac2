"""Outputs that a caller gives to the calls on a model's table and head: none that stands in an autograd graph, whose history would stay and go through what has been
overwritten."""
import pytest
import torch

import paper_2506_03887_amd as P
from test_matrices_arguments import EMBED, LOGITS, zeros

CALLS = [("embed", EMBED, (4, 6)), ("head_logits", LOGITS, (4, 40))]


@pytest.mark.parametrize("call,good,shape", CALLS)
def test_an_output_with_a_history_is_refused(call, good, shape):
    leaf = zeros(*shape).requires_grad_()
    for out in (leaf, leaf * 2, (leaf * 2).detach().requires_grad_()):
        with pytest.raises(AssertionError, match="out: not part of an autograd graph"):
            getattr(P, call)(**good, out=out)
    with torch.no_grad(), pytest.raises(TypeError):                # (as far as tensors in host memory get)
        getattr(P, call)(**good, out=leaf)


@pytest.mark.gpu
def test_outputs_without_a_history_are_written():
    weight, tokens = torch.randn(9, 6, device="cuda"), torch.tensor([3, -1, 8], device="cuda")
    out = torch.full((3, 6), 9.0, device="cuda")
    assert P.embed(weight, tokens, out=out) is not None and torch.equal(out[0], weight[3]) and not out[1].any()
    with torch.no_grad():                                          # as torch's own operations take it there
        kept = torch.full((3, 6), 9.0, device="cuda").requires_grad_()
        P.embed(weight, tokens, out=kept)
    assert torch.equal(kept.detach(), out)
