"""On-policy distillation under a grammar: a student writes text that the grammar allows, a teacher says for every position which of the
allowed tokens it finds best, and the student is taught these lists.

Teacher and student are the smallest language models there are (a table of logits by the last token, the student's of low rank), so
that the whole loop is the library's calls:

  every step        apply_mask_sample      the student's token, drawn behind the mask by temperature and top-p
                    apply_mask_topk        the teacher's k best allowed tokens at the same place
                    advance_fill_mask      the texts advance, the next masks
  every so often    distill_loss           through autograd into the student's factors, or
                    distill_loss_grad      loss and gradient at once, handed on by hand

python examples/distill_constrained.py [--pass]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2506_03887_amd import Pre3, distill_loss, distill_loss_grad  # noqa: E402
from workloads import grammars, vocab as vocabularies  # noqa: E402


class Texts:
    """A batch of texts under a grammar: their parse stacks, and the mask of the next token of each."""

    def __init__(self, lib, batch, cap=256):
        dev = torch.device("cuda")
        start = lib.initial_state(0)
        self.lib, self.batch = lib, batch
        self.states = torch.full((batch,), start, dtype=torch.int32, device=dev)
        self.data = torch.full((batch, cap), start, dtype=torch.int32, device=dev)
        self.length = torch.ones(batch, dtype=torch.int32, device=dev)
        self.err = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.mask = torch.empty((batch, lib.words), dtype=torch.int32, device=dev)
        lib.bind_state(self.states, self.data, self.length, self.err)
        lib.fill_mask(self.states, self.data, self.length, self.mask)


def collect(texts, student, teacher, last, steps, k, generator, temperature, top_p):
    """`steps` tokens of every text, written by the student: where they were written (the last tokens before them), the masks and the
    teacher's lists there."""
    lib, batch, dev = texts.lib, texts.batch, last.device
    seen = torch.empty((steps, batch), dtype=torch.int64, device=dev)
    masks = torch.empty((steps, batch, lib.words), dtype=torch.int32, device=dev)
    ids = torch.empty((steps, batch, k), dtype=torch.int32, device=dev)
    values = torch.empty((steps, batch, k), dtype=torch.bfloat16, device=dev)
    token = torch.empty(batch, dtype=torch.int32, device=dev)
    logprob = torch.empty((steps, batch), device=dev)
    for t in range(steps):
        seen[t], masks[t] = last, texts.mask
        with torch.no_grad():
            lib.apply_mask_topk(teacher[last], texts.mask, ids[t], values[t])
            uniform = torch.rand(batch, generator=generator, device=dev)
            lib.apply_mask_sample(student(last), texts.mask, uniform, token, logprob[t], temperature=temperature, top_p=top_p)
        lib.advance_fill_mask(token, texts.mask, restart_on_eos=True)
        last = token.long()
    return seen.flatten(), masks.flatten(0, 1), ids.flatten(0, 1), values.flatten(0, 1), logprob, last


def train(vocab=4096, batch=64, steps=16, rounds=20, k=32, rank=64, tau=1.0, one_pass=False, seed=1, report=print):
    """The mean loss of every round."""
    dev = torch.device("cuda")
    generator = torch.Generator(device=dev).manual_seed(seed)
    words = vocabularies.bpe_like_vocab(vocab, 16, seed)
    lib = Pre3(grammars.JSON, words.bytes, words.offsets, words.eos_id, stack_cap=256)
    teacher = (3 * torch.randn((vocab, vocab), generator=generator, device=dev)).bfloat16()
    left = (torch.randn((vocab, rank), generator=generator, device=dev) / rank ** 0.5).requires_grad_()
    right = torch.randn((rank, vocab), generator=generator, device=dev).requires_grad_()
    optimizer = torch.optim.Adam([left, right], lr=0.05)

    def student(last):
        return (left[last] @ right).bfloat16()

    texts = Texts(lib, batch)
    last = torch.zeros(batch, dtype=torch.int64, device=dev)
    temperature, top_p = torch.full((batch,), 0.9, device=dev), torch.full((batch,), 0.95, device=dev)
    losses = []
    for r in range(rounds):
        seen, masks, ids, values, logprob, last = collect(texts, student, teacher, last, steps, k, generator, temperature, top_p)
        optimizer.zero_grad()
        logits = student(seen)
        if one_pass:
            weight = torch.full((len(seen),), 1 / len(seen), device=dev)
            loss, grad = distill_loss_grad(logits, ids, values, masks, temperature=tau, row_weight=weight)
            loss = loss.mean()
            logits.backward(grad)
        else:
            loss = distill_loss(logits, ids, values, masks, temperature=tau).mean()
            loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))
        report(f"round {r}: loss {losses[-1]:.4f}, log-probability of the student's tokens {float(logprob.mean()):.3f}")
    assert not texts.err.any(), "a drawn token was not allowed"
    return losses


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    parser.add_argument("--pass", dest="one_pass", action="store_true", help="loss and gradient in one pass")
    train(one_pass=parser.parse_args().one_pass)
