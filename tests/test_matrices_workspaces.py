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
