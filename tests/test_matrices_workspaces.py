"""What the calls on a model's table and head say of their workspaces (host code: no GPU needed)."""
import ctypes as c
import itertools

import pytest

from test_matrices_arguments import NOWHERE, Head, lib

SIZES = list(itertools.product((0, 1, 2), (1, 5, 40, 140, 3000), (7, 5000, 128256, 500001), (8, 1001, 4097)))


def head(kind, rows, vocab, dim):
    return Head(NOWHERE, NOWHERE, NOWHERE, None, dim, dim, kind, 4, rows, vocab, dim, NOWHERE, 0)


@pytest.mark.parametrize("kind,rows,vocab,dim", [*SIZES, (0, 40, 500001, 1001), (2, 82432, 100, 1024)])
def test_a_workspace_with_gradients_serves_the_loss_as_well(kind, rows, vocab, dim):
    h = head(kind, rows, vocab, dim)
    loss, gradients = (lib().pre3_head_workspace_bytes(c.byref(h), x) for x in (0, 1))
    assert 0 < loss <= gradients


@pytest.mark.parametrize("kind,rows,vocab,dim,most", [(2, 16, 128256, 2048, 32), (1, 40, 100003, 1001, 32), (2, 64, 128256, 4096, 64)])
def test_a_loss_alone_from_weights_as_they_lie_takes_no_room_for_packed_ones(kind, rows, vocab, dim, most):
    """In MiB: the logits, their parts and the hidden states."""
    h = head(kind, rows, vocab, dim)
    loss, alone = (lib().pre3_head_workspace_bytes(c.byref(h), x) for x in (0, 2))
    assert 0 < alone <= most << 20 and alone < loss
    h.workspace_bytes = alone - 1
    assert lib().pre3_head_loss(c.byref(h), NOWHERE, None, None) == -1


@pytest.mark.parametrize("kind,rows,vocab,dim", SIZES)
def test_a_loss_alone_takes_no_more_than_one_that_leaves_something(kind, rows, vocab, dim):
    h = head(kind, rows, vocab, dim)
    loss, alone = (lib().pre3_head_workspace_bytes(c.byref(h), x) for x in (0, 2))
    assert 0 < alone <= loss
