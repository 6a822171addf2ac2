"""The table and the head together, as a model has them: a training step whose table is its head as well, and steps of constrained decoding with a
head in 8 bits."""
import math
import os
import sys

import pytest
import torch

from test_gpu_head8 import quantised
from test_gpu_head_loss import TYPES, close, inputs, pack, reference

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,vocab,dim", [("bf16", 6, 700, 64), ("f16", 90, 1003, 129), ("f32", 40, 513, 64), ("bf16", 300, 2001, 256)])
def test_a_step_whose_table_is_its_head(dtype, rows, vocab, dim):
    """loss(embed(E, tokens, 2), E): the gradient of E is the head's and the table's.  A row is exact (a power of two), so the loss and the head's gradients
    are off as in their own tests; the table's gradient sums rows of d hidden, each off by its own, with sums in 32 bits ((n + 2) * 2^-24 of their
    absolute values) and half a step; the two are added by torch: half a step more."""
    from paper_2506_03887_amd import embed, head_loss
    _, weight, targets, allowed, g = inputs(dtype, rows, vocab, dim, "mixed", seed=rows)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    tokens = torch.randint(-1, vocab // 4, (rows,), generator=gen, device="cuda")
    bits = pack(allowed)
    table = weight.detach().requires_grad_()
    hidden = embed(table, tokens, 2.0)
    hidden.retain_grad()
    loss = head_loss(hidden, table, targets, bits)
    loss.backward(g)
    there = tokens >= 0
    exact_rows = (2 * weight.double()[tokens.clamp(min=0)]) * there[:, None]
    assert torch.equal(hidden.detach().double(), exact_rows)
    want_loss, (d_h, off_h), (d_w, off_w) = reference(hidden.detach(), weight, targets, allowed, g, dtype)
    close(loss.detach(), want_loss, "loss")
    close(hidden.grad, (d_h, off_h), "hidden")
    half, tiny = torch.finfo(TYPES[dtype]).eps / 2, torch.finfo(TYPES[dtype]).tiny * 2.0 ** -8
    sums, off, size = (torch.zeros((vocab, dim), dtype=torch.float64, device="cuda").index_add_(0, tokens[there], 2 * x[there]) for x in (d_h, off_h, d_h.abs() + off_h))
    n = torch.bincount(tokens[there], minlength=vocab).double()[:, None]
    off = off + (n + 2) * 2.0 ** -24 * size
    off = off + half * (sums.abs() + off) + tiny
    total = sums + d_w
    close(table.grad, (total, off + off_w + half * (total.abs() + off + off_w) + tiny), "table")


def test_steps_of_decoding():
    """embed, head_logits behind the mask, the sampler, the masks of the texts: the step by itself against plain products, and in a graph."""
    from examples.distill_constrained import Texts
    from paper_2506_03887_amd import Pre3, embed, head_logits, quantise_rows
    from workloads import grammars, vocab as vocabularies
    vocab, batch, dim, steps = 1024, 16, 96, 12
    gen = torch.Generator(device="cuda").manual_seed(3)
    words = vocabularies.bpe_like_vocab(vocab, 16, 1)
    table = torch.randn((vocab, dim), generator=gen, device="cuda").bfloat16()
    weight, scale = quantise_rows(torch.randn((vocab, dim), generator=gen, device="cuda"))
    uniform = torch.rand((steps, batch), generator=gen, device="cuda")

    def run(captured):
        lib = Pre3(grammars.JSON, words.bytes, words.offsets, words.eos_id, stack_cap=256)
        texts = Texts(lib, batch)
        token, draw = torch.full((batch,), -1, dtype=torch.int32, device="cuda"), torch.empty(batch, device="cuda")
        hidden, logits = torch.empty((batch, dim), dtype=torch.bfloat16, device="cuda"), torch.empty((batch, vocab), dtype=torch.bfloat16, device="cuda")

        def choose():
            embed(table, token, 0.5, out=hidden)
            head_logits(hidden, weight, scale, texts.mask, out=logits)
            lib.apply_mask_sample(logits, texts.mask, draw, token, temperature=warm, top_p=most)

        def advance():
            lib.advance_fill_mask(token, texts.mask, restart_on_eos=True)

        warm, most = torch.full((batch,), 0.9, device="cuda"), torch.full((batch,), 0.95, device="cuda")
        graph = None
        if captured:
            draw.copy_(uniform[0])
            choose()                                                # (all workspaces are there)
            token.fill_(-1)
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                choose()
        seen = []
        for t in range(steps):
            draw.copy_(uniform[t])
            before, mask = token.long(), texts.mask.clone()
            choose() if graph is None else graph.replay()
            allowed = (mask[:, torch.arange(vocab, device="cuda") // 32] >> (torch.arange(vocab, device="cuda") % 32) & 1).bool()
            row = (0.5 * table.double()[before.clamp(min=0)]) * (before >= 0)[:, None]
            assert torch.equal(hidden.double(), row)
            q, s = quantised(hidden)
            exact = (q @ weight.double().T) * s.double()[:, None] * scale.double()
            assert (logits[~allowed] == -math.inf).all()
            assert ((logits.double() - exact).abs()[allowed] <= (2.0 ** -8 + 3 * 2.0 ** -24) * exact.abs()[allowed]).all()
            assert allowed[torch.arange(batch, device="cuda"), token.long()].all()
            seen.append(token.clone())
            advance()
        assert not texts.err.any()
        return torch.stack(seen)

    assert torch.equal(run(False), run(True))
