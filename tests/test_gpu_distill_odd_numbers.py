"""The distillation where numbers are not finite, against the definition: a token is open if it is allowed and its logit is not -inf,
an entry counts if its token is open and the teacher's logit is not -inf, and NaNs among the open logits or the list come out as
NaN; what is not open has the gradient 0, whatever the rest of its row or the row's weight is."""
import math

import numpy as np
import pytest
import torch

from paper_2506_03887_amd import distill_loss, distill_loss_grad
from test_gpu_distill import LOG_Z, check_grad, pack
from workloads.vocab import BASE_SEED

pytestmark = pytest.mark.gpu

# one wave; 256, 512 and 1,024 threads; a row over several blocks
FORMS = [(6, 7, torch.float32), (6, 1003, torch.bfloat16), (5, 8200, torch.float16), (5, 20011, torch.float32), (200, 60003, torch.bfloat16),
         (260, 28011, torch.float32), (4, 100003, torch.float16), (3, 128256, torch.float32)]


def reference(x, ids, values, bits, tau, weight):
    """(loss, gradient, open tokens, rows with an entry) in 64 bits on the CPU."""
    x, ids, values, weight = x.detach().double().cpu(), ids.cpu().long(), values.double().cpu(), weight.double().cpu()
    is_open = bits & (x != -math.inf)
    at = ids.clamp(0, x.shape[1] - 1)
    entry = (ids == at) & is_open.gather(1, at) & (values != -math.inf)
    live = entry.any(1)
    logp = torch.log_softmax(torch.where(is_open, x / tau, torch.full_like(x, -math.inf)), dim=1)
    logq = torch.log_softmax(torch.where(entry, values / tau, torch.full_like(values, -math.inf)), dim=1)
    q = torch.where(entry, logq.exp(), torch.zeros_like(logq))
    loss = tau * tau * torch.where(entry, q * (logq - logp.gather(1, at)), torch.zeros_like(q)).sum(1)
    p, target = logp.exp(), torch.zeros_like(x).scatter_add_(1, at, q)
    some = is_open & live[:, None]
    grad = torch.where(some, weight[:, None] * tau * (p - target), torch.zeros_like(x))
    return torch.where(live, loss, torch.zeros_like(loss)), grad, p, target, is_open, live


def everything(x, ids, values, mask, weight, tau):
    """Loss and gradient by every way to them."""
    leaf = x.detach().clone().requires_grad_()
    loss = distill_loss(leaf, ids, values, mask, temperature=tau)
    grad, = torch.autograd.grad(loss, leaf, weight)
    yield loss.detach(), grad
    yield distill_loss_grad(x, ids, values, mask, temperature=tau, row_weight=weight)
    place = x.clone()
    yield distill_loss_grad(place, ids, values, mask, temperature=tau, row_weight=weight, out=place)


def kind(t):
    """NaN, the infinities, zero, other numbers."""
    t = t.double().cpu()
    return torch.where(torch.isnan(t), 4, torch.where(torch.isinf(t), 2 + t.sign().nan_to_num(), (t != 0).double())).int()


def inputs(rng, rows, vocab, dtype, k=3):
    """Finite rows, each with k different tokens listed."""
    x = torch.as_tensor(rng.normal(size=(rows, vocab)) * 2).to(dtype).cuda()
    ids = torch.stack([torch.as_tensor(rng.permutation(vocab)[:k]) for _ in range(rows)]).int().cuda()
    return x, ids, torch.as_tensor(rng.normal(size=(rows, k))).float().cuda()


@pytest.mark.parametrize("rows,vocab,dtype", FORMS)
def test_a_nan_among_a_handful_of_allowed_tokens(rows, vocab, dtype):
    """Two to five allowed tokens, mostly one to a thread, the NaN not among the listed ones; a row of nothing but the NaN allowed and listed
    tokens that are not."""
    rng = np.random.default_rng(BASE_SEED + 37 + vocab)
    x, ids, values = inputs(rng, rows, vocab, dtype, k=1)
    bits = torch.zeros((rows, vocab), dtype=torch.bool)
    odd = torch.zeros(rows, dtype=torch.int64)
    for b in range(rows):
        others = [t for t in rng.permutation(vocab)[:8] if t != int(ids[b])]
        bits[b, others[:1 + b % 4]] = True
        bits[b, int(ids[b])] = True
        odd[b] = int(others[0]) if b % 2 == 0 else vocab - 1 if int(ids[b]) != vocab - 1 else 0
    bits[torch.arange(rows), odd] = True
    bits[0] = False
    bits[0, odd[0]] = True                                   # the listed token is not allowed: no entry, whatever the NaN
    x[torch.arange(rows), odd.cuda()] = math.nan
    weight = torch.ones(rows, device="cuda")
    loss_want, grad_want, *_ = reference(x, ids, values, bits, 2.0, weight)
    assert loss_want[0] == 0 and torch.isnan(loss_want[1:]).all()
    for loss, grad in everything(x, ids, values, pack(bits).cuda(), weight, 2.0):
        assert torch.equal(torch.isnan(loss.cpu()), torch.isnan(loss_want)) and loss[0] == 0
        assert torch.isnan(grad.cpu()[bits & (torch.arange(rows) > 0)[:, None]]).all() and (grad[0] == 0).all()


@pytest.mark.parametrize("rows,vocab,dtype", FORMS)
def test_a_listed_token_with_a_nan(rows, vocab, dtype):
    """A student of nothing but NaNs, of NaNs where the teacher lists something, and at one of the listed tokens."""
    rng = np.random.default_rng(BASE_SEED + 31 + vocab)
    x, ids, values = inputs(rng, rows, vocab, dtype)
    x[0] = math.nan
    x[1, ids[1].long()] = math.nan
    x[2, ids[2, 1].long()] = math.nan
    weight, spread = torch.ones(rows, device="cuda"), float((x[3:].max() - x[3:].min()) / 1.5 * 1.45) if rows > 3 else 0.0
    loss_want, grad_want, *rest = reference(x, ids, values, torch.ones(x.shape, dtype=torch.bool), 1.5, weight)
    assert torch.isnan(loss_want[:3]).all() and torch.isnan(grad_want[:3]).all()
    for loss, grad in everything(x, ids, values, None, weight, 1.5):
        assert torch.equal(torch.isnan(loss.cpu()), torch.isnan(loss_want))
        assert torch.equal(torch.isnan(grad.cpu()), torch.isnan(grad_want))
        assert ((loss[3:].double().cpu() - loss_want[3:]).abs() <= 1.5 ** 2 * LOG_Z + loss_want[3:].abs() * 2.0 ** -23).all()
        check_grad(grad[3:], *(r[3:] for r in rest), weight[3:].double().cpu(), 1.5, spread)


@pytest.mark.parametrize("rows,vocab,dtype", FORMS)
def test_what_is_not_open_has_no_gradient(rows, vocab, dtype):
    """Whole groups of masked tokens, logits of -inf, and both in groups with open ones: zero beside NaNs and +inf in the row, and under
    weights that are infinite, NaN or zero."""
    rng = np.random.default_rng(BASE_SEED + 41 + vocab)
    x, ids, values = inputs(rng, rows, vocab, dtype, k=2)
    bits = torch.as_tensor(rng.random((rows, vocab)) < 0.5)
    bits[:, vocab // 4:vocab // 2] = False
    x[:, vocab // 2::3] = -math.inf
    for b in range(rows):                                    # what is listed is open, and so is the odd one
        at = torch.cat([ids[b].long().cpu(), torch.tensor([b % 4])])
        bits[b, at] = True
        x[b, at.cuda()] = x[b, at.cuda()].clamp(-3, 3).nan_to_num()
    weight = torch.ones(rows, device="cuda")
    x[0, 0], x[1, 1] = math.nan, math.inf
    weight[2] = math.inf
    if rows > 3:
        weight[3] = math.nan
    if rows > 4:
        weight[4] = 0.0
    loss_want, grad_want, _, _, is_open, live = reference(x, ids, values, bits, 1.0, weight)
    assert live.all() and (grad_want[~is_open] == 0).all()
    for loss, grad in everything(x, ids, values, pack(bits).cuda(), weight, 1.0):
        assert torch.equal(torch.isnan(loss.cpu()), torch.isnan(loss_want))
        assert (grad.cpu()[~is_open] == 0).all()
        assert torch.equal(kind(grad)[:5], kind(grad_want)[:5])
