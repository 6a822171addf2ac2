"""Forward-mode tangents, which the calls on a model's table and head would lose, are refused before anything else is looked at (no GPU needed)."""
import pytest
import torch
import torch.autograd.forward_ad as fwd

import paper_2506_03887_amd as P
from test_matrices_arguments import EMBED, HEAD, LOGITS, zeros

CALLS = [("embed", EMBED, "weight"), ("head_loss", HEAD, "hidden"), ("head_loss", HEAD, "weight"), ("head_loss_grad", HEAD, "hidden"), ("head_loss_grad", HEAD, "weight"),
         ("head_loss_grad", dict(HEAD, row_weight=zeros(4)), "row_weight"), ("quantise_rows", dict(x=zeros(4, 6)), "x"), ("head_logits", LOGITS, "hidden"), ("head_logits", LOGITS, "scale")]


@pytest.mark.parametrize("call,good,name", CALLS)
def test_a_tangent_is_refused(call, good, name):
    with fwd.dual_level():
        x = good[name]
        with pytest.raises(NotImplementedError, match="no forward-mode derivative"):
            getattr(P, call)(**{**good, name: fwd.make_dual(x, torch.ones_like(x))})
