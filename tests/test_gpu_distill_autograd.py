"""What autograd knows of the distillation's calls: writes in place, and forward mode."""
import pytest
import torch

from paper_2506_03887_amd import distill_loss, distill_loss_grad
from workloads.vocab import BASE_SEED

pytestmark = pytest.mark.gpu


def inputs(rows=12, vocab=1003, k=8):
    gen = torch.Generator(device="cuda").manual_seed(BASE_SEED + 43)
    ids = torch.randint(vocab, (rows, k), generator=gen, device="cuda", dtype=torch.int32)
    values = torch.randn((rows, k), generator=gen, device="cuda")
    hidden, head = torch.randn((rows, 16), generator=gen, device="cuda"), torch.randn((16, vocab), generator=gen, device="cuda")
    return hidden.requires_grad_(), head.requires_grad_(), ids, values


def test_a_gradient_in_place_of_saved_logits_is_an_error_of_their_backward_pass():
    hidden, head, ids, values = inputs()
    logits = hidden @ head
    loss = distill_loss(logits, ids, values)                 # saves its logits
    distill_loss_grad(logits, ids, values, out=logits)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()
    logits = 30 * torch.tanh(hidden @ head)                  # the product's factor is saved, not the product
    capped = torch.tanh(hidden @ head)                       # saves what it returns
    for x, raises in ((logits, False), (capped, True)):
        _, grad = distill_loss_grad(x, ids, values, out=x)
        if raises:
            with pytest.raises(RuntimeError, match="modified by an inplace operation"):
                x.backward(grad)
        else:
            x.backward(grad)


def test_a_part_of_a_saved_tensor():
    hidden, head, ids, values = inputs()
    wide = torch.exp(hidden @ head)                          # saves what it returns
    distill_loss_grad((hidden @ head).detach(), ids, values, out=wide.detach()[:, :1003])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        wide.sum().backward()


def test_a_gradient_in_place_that_is_handed_on():
    hidden, head, ids, values = inputs()
    want = torch.autograd.grad(distill_loss(hidden @ head, ids, values).sum(), (hidden, head))
    logits = hidden @ head                                   # a product saves its factors alone
    _, grad = distill_loss_grad(logits, ids, values, out=logits)
    logits.backward(grad)
    assert torch.equal(hidden.grad, want[0]) and torch.equal(head.grad, want[1])


def test_tensors_made_in_inference_mode():
    hidden, head, ids, values = inputs()
    with torch.inference_mode():
        x = hidden @ head
        loss, grad = distill_loss_grad(x, ids, values)
    plain = x.clone()
    again, same = distill_loss_grad(x, ids, values, out=x)
    assert torch.equal(loss, again) and torch.equal(grad, same) and same is x
    assert torch.equal(distill_loss(plain, ids, values), loss)
    with torch.inference_mode():
        distill_loss_grad(plain, ids, values, out=plain)


def test_forward_mode_is_refused():
    """A tangent of the logits, or of the teacher's, would be lost: the loss would read as constant."""
    import torch.autograd.forward_ad as forward
    hidden, head, ids, values = inputs()
    logits = (hidden @ head).detach()
    for needs in (False, True):
        with forward.dual_level():
            dual = forward.make_dual(logits.clone().requires_grad_(needs), torch.ones_like(logits))
            with pytest.raises(NotImplementedError, match="forward-mode"):
                distill_loss(dual, ids, values)
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                distill_loss(dual, ids, values)
            with pytest.raises(NotImplementedError, match="forward-mode"):
                distill_loss(logits, ids, forward.make_dual(values, torch.ones_like(values)))
            primal = forward.unpack_dual(dual).primal
            assert torch.equal(distill_loss(primal.detach(), ids, values), distill_loss(logits, ids, values))
    with pytest.raises(RuntimeError):
        torch.func.jvp(lambda x: distill_loss(x, ids, values), (logits,), (torch.ones_like(logits),))


def test_a_mask_that_the_next_step_has_overwritten_is_an_error():
    """A loop that keeps one mask for all steps and goes backward at its end."""
    import numpy as np
    from paper_2506_03887_amd import Pre3
    hidden, head, ids, values = inputs()
    rows, vocab = 12, 1003
    text = np.append(np.resize(np.frombuffer(b"abcde", dtype=np.uint8), vocab - 1), np.uint8(0))
    lib = Pre3("S ::= S X | X\nX ::= [a-e]\n", text, np.append(np.arange(vocab), vocab - 1), vocab - 1, stack_cap=8)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    states, data, length, mask = i32(rows) + lib.initial_state(0), i32(rows, 8) + lib.initial_state(0), i32(rows) + 1, i32(rows, lib.words)
    lib.bind_state(states, data, length, i32(rows))
    lib.fill_mask(states, data, length, mask)
    loss = distill_loss(hidden @ head, ids, values, mask)
    loss.sum().backward(retain_graph=True)
    lib.advance_fill_mask(i32(rows), mask)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()
