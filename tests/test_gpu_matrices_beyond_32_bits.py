"""Tables, heads and logits of more than 2^31 numbers and 2^32 bytes, against the definition in 64 bits taken in stretches of tokens, within the bounds that
test_gpu_head_loss, test_gpu_embed and test_gpu_head8 derive (weights of a variance of 4 / dim, hidden states of 1 and more)."""
import math

import pytest
import torch

from test_gpu_head_loss import TYPES, U, close

pytestmark = pytest.mark.gpu
STRETCH = 1 << 16


def numbers(rows, dim, dtype, gen, scale=1.0):
    """[rows, dim], made in stretches."""
    x = torch.empty((rows, dim), dtype=dtype, device="cuda")
    for lo in range(0, rows, STRETCH):
        x[lo:lo + STRETCH] = torch.randn((min(STRETCH, rows - lo), dim), generator=gen, device="cuda") * scale
    return x


@pytest.mark.parametrize("rows,dim", [(2, 2048), (2, 2047), (40, 2048), (40, 2047), (150, 2048)])
def test_heads(rows, dim):
    from paper_2506_03887_amd import head_loss, head_loss_grad
    vocab, r = 1_100_001, 2.0 ** -8
    assert vocab * dim > 2 ** 31 and 2 * vocab * dim > 2 ** 32
    print(f"[head] {rows} x {vocab} x {dim}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(dim + rows)
    weight = numbers(vocab, dim, torch.bfloat16, gen, 2 / math.sqrt(dim))
    targets = torch.randint(vocab, (rows,), generator=gen, device="cuda")
    targets[0], targets[1] = vocab - 1, 5
    hidden = (torch.randn((rows, dim), generator=gen, device="cuda") + 1.5 * weight[targets].float()).bfloat16()
    g = torch.rand(rows, generator=gen, device="cuda") + 0.5
    loss, d_h, d_w = head_loss_grad(hidden, weight, targets, row_weight=g)
    alone = head_loss(hidden, weight, targets)
    h, g64 = hidden.double(), g.double()[:, None]
    # two passes over the tokens: the rows' sums and largest errors, then the gradients
    x = torch.empty((rows, vocab), dtype=torch.float64, device="cuda")
    size = torch.zeros((rows, 1), dtype=torch.float64, device="cuda")
    for lo in range(0, vocab, STRETCH):
        w = weight[lo:lo + STRETCH].double()
        x[:, lo:lo + STRETCH] = h @ w.T
        size = torch.maximum(size, (h.abs() @ w.abs().T).amax(dim=1, keepdim=True))
    e = (dim + 16) * U * size
    logp = torch.log_softmax(x, dim=1)
    want = -logp[torch.arange(rows, device="cuda"), targets]
    off = 2 * e[:, 0] + 2.0 ** -16 + 2.0 ** -23 * want.abs()
    close(loss, (want, off), "loss")
    close(alone, (want, off), "loss alone")
    s = torch.exp(logp)
    off_s = s * (2 * e + 2.0 ** -16)
    s[torch.arange(rows, device="cuda"), targets] -= 1
    off_s = g64 * (off_s + (r + 2.0 ** -20) * s.abs())
    s *= g64
    half, tiny = r, torch.finfo(torch.bfloat16).tiny * 2.0 ** -8
    sums = [torch.zeros((rows, dim), dtype=torch.float64, device="cuda") for _ in range(3)]
    for lo in range(0, vocab, STRETCH):
        w, s_l, off_l = weight[lo:lo + STRETCH].double(), s[:, lo:lo + STRETCH], off_s[:, lo:lo + STRETCH]
        for total, term in zip(sums, (s_l @ w, off_l @ w.abs(), s_l.abs() @ w.abs())):
            total += term
        exact = s_l.T @ h
        off_w = off_l.T @ h.abs() + (rows + 16) * U * (s_l.abs().T @ h.abs())
        close(d_w[lo:lo + STRETCH], (exact, off_w * (1 + half) + half * exact.abs() + tiny), f"weight from {lo}")
    close(d_h, (sums[0], (sums[1] + (vocab + 16) * U * sums[2]) * (1 + half) + half * sums[0].abs() + tiny), "hidden")


def test_a_table_and_its_gradient():
    from paper_2506_03887_amd import embed
    vocab, dim, rows = 1 << 22, 520, 2000
    gen = torch.Generator(device="cuda").manual_seed(1)
    table = numbers(vocab, dim, torch.float16, gen).requires_grad_()
    assert table.numel() > 2 ** 31
    tokens = torch.randint(vocab - 500, vocab, (rows,), generator=gen, device="cuda")
    tokens[:3] = torch.tensor([0, vocab - 1, -1], device="cuda")
    out = embed(table, tokens)
    some = tokens >= 0
    assert torch.equal(out[some], table.detach()[tokens[some]]) and not out[2].any()
    upstream = torch.randn((rows, dim), generator=gen, device="cuda").half()
    grad, = torch.autograd.grad(out, table, upstream)
    last = vocab - 500
    places = torch.where(tokens >= last, tokens - last, 500)
    exact, size = (torch.zeros((501, dim), dtype=torch.float64, device="cuda").index_add_(0, places, x) for x in (upstream.double(), upstream.double().abs()))
    n = torch.bincount(places, minlength=501).double()[:, None]
    half = 2.0 ** -11 + 2.0 ** -23
    off = (n + 2) * U * size * (1 + half) + half * exact.abs() + torch.finfo(torch.float16).tiny * 2.0 ** -8
    assert ((grad[last:].double() - exact[:500]).abs() <= off[:500]).all()
    assert torch.equal(grad[0], upstream[0])
    for lo in range(1, last, 1 << 19):
        assert not grad[lo:min(lo + (1 << 19), last)].any()


def test_logits_in_8_bits():
    from paper_2506_03887_amd import head_logits, quantise_rows
    gen = torch.Generator(device="cuda").manual_seed(2)
    for rows, vocab, dim in ((2100, 1_048_577, 24), (2, 2_097_152, 2064)):
        assert rows * vocab > 2 ** 31 or vocab * dim > 2 ** 32
        print(f"[head8] {rows} x {vocab} x {dim}", flush=True)
        x = numbers(vocab, dim, torch.bfloat16, gen)
        weight, scale = quantise_rows(x)
        last = x[-3:].double()
        top = last.abs().amax(dim=1, keepdim=True)
        assert torch.equal(weight[-3:].double(), torch.round((last * (127 / top).float().double()).float()).double()) and torch.equal(scale[-3:], (top[:, 0] / 127).float())
        hidden = torch.randn((rows, dim), generator=gen, device="cuda").bfloat16()
        q, s = quantise_rows(hidden)
        logits = head_logits(hidden, weight, scale)
        for r in sorted({0, 1, rows // 2, rows - 1}):
            for lo in range(0, vocab, STRETCH):
                exact = (weight[lo:lo + STRETCH].double() @ q[r].double()) * s[r].double() * scale[lo:lo + STRETCH].double()
                assert ((logits[r, lo:lo + STRETCH].double() - exact).abs() <= (2.0 ** -8 + 3 * U) * exact.abs() + torch.finfo(torch.bfloat16).tiny).all(), (r, lo)
        del x, weight, logits


@pytest.mark.parametrize("vocab", [40, 300])
def test_hidden_states(vocab):
    """As many rows as are taken; the gradient of the weights is a sum over all of them."""
    from paper_2506_03887_amd import head_loss_grad
    rows, dim, r = 1 << 20, 2064, 2.0 ** -8
    print(f"[head] {rows} x {vocab} x {dim}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    weight = numbers(vocab, dim, torch.bfloat16, gen, 2 / math.sqrt(dim))
    hidden = numbers(rows, dim, torch.bfloat16, gen)
    assert hidden.numel() > 2 ** 31
    targets = torch.randint(-1, vocab, (rows,), generator=gen, device="cuda")
    targets[-1] = vocab - 1
    loss, d_h, d_w = head_loss_grad(hidden, weight, targets)
    w, tiny = weight.double(), torch.finfo(torch.bfloat16).tiny * 2.0 ** -8
    sums = [torch.zeros((vocab, dim), dtype=torch.float64, device="cuda") for _ in range(3)]
    for lo in range(0, rows, STRETCH):
        h, t = hidden[lo:lo + STRETCH].double(), targets[lo:lo + STRETCH]
        some, at = t >= 0, torch.arange(len(t), device="cuda")
        e = (dim + 16) * U * (h.abs() @ w.abs().T).amax(dim=1, keepdim=True)
        logp = torch.log_softmax(h @ w.T, dim=1)
        want = -logp[at, t.clamp(0)] * some
        close(loss[lo:lo + STRETCH], (want, (2 * e[:, 0] + 2.0 ** -16 + 2.0 ** -23 * want) * some), f"loss from {lo}")
        s = torch.exp(logp)
        off_s = s * (2 * e + 2.0 ** -16)
        s[at, t.clamp(0)] -= 1
        off_s, s = (off_s + (r + 2.0 ** -20) * s.abs()) * some[:, None], s * some[:, None]
        exact = s @ w
        off = off_s @ w.abs() + (vocab + 16) * U * (s.abs() @ w.abs())
        close(d_h[lo:lo + STRETCH], (exact, off * (1 + r) + r * exact.abs() + tiny), f"hidden from {lo}")
        for total, term in zip(sums, (s.T @ h, off_s.T @ h.abs(), s.abs().T @ h.abs())):
            total += term
    close(d_w, (sums[0], (sums[1] + (rows + 16) * U * sums[2]) * (1 + r) + r * sums[0].abs() + tiny), "weight")
