"""distill_loss, its backward pass and distill_loss_grad against their formulas in 64 bits, and the gradient against differences.

Tolerances, from how the kernels compute.  x = logit * scale - top is one rounded operation (and scale a rounded number), so a weight
2^x is off by |x| 2^-24 ln 2 twice and by an ulp of the exponential, 2^-23; weighted by p, |x| is at most log2 of the vocabulary and
the entropy, 36 for 2^18 tokens; a sum of 32 bits over one thread's tokens adds 2^-24 for each of at most 256.  A row's log Z is then
off by less than (2 * 36 * 0.7 + 2 + 256) 2^-24 < 2^-15, and so is a loss / tau^2.  A gradient is p - q with p off by that and by its own
|x|, rounded once to its type; below the type's smallest number it is what the type has."""
import math

import numpy as np
import pytest
import torch

from paper_2506_03887_amd import Pre3, distill_loss, distill_loss_grad
from workloads import grammars as G
from workloads.vocab import BASE_SEED

pytestmark = pytest.mark.gpu

DTYPES = (torch.bfloat16, torch.float16, torch.float32)
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
SMALLEST = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24, torch.float32: 2.0 ** -126}
LOG_Z = 2.0 ** -15


def unpack(mask, vocab):
    bits = (mask.unsqueeze(2) >> torch.arange(32, dtype=torch.int32)) & 1
    return bits.reshape(mask.shape[0], -1)[:, :vocab].bool()


def pack(bits):
    rows, vocab = bits.shape
    x = torch.zeros((rows, -(-vocab // 32) * 32), dtype=torch.int64)
    x[:, :vocab] = bits
    x = (x.view(rows, -1, 32) << torch.arange(32)).sum(2)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).int()


def reference(x, ids, values, mask, tau):
    """(loss, p, target, open tokens, live rows) in 64 bits on the CPU."""
    x, ids, values = x.detach().double().cpu(), ids.cpu().long(), values.double().cpu()
    rows, vocab = x.shape
    is_open = ~(x == -math.inf)
    if mask is not None:
        is_open &= unpack(mask.cpu(), vocab)
    inside = (ids >= 0) & (ids < vocab)
    at = torch.where(inside, ids, torch.zeros_like(ids))
    ok = inside & is_open.gather(1, at) & ~(values == -math.inf) & ~torch.isnan(x.gather(1, at))
    live = ok.any(1)
    logp = torch.log_softmax(torch.where(is_open, x / tau, torch.full_like(x, -math.inf)), dim=1)
    t = torch.where(ok | ~live[:, None], values / tau, torch.full_like(values, -math.inf))
    logq = torch.log_softmax(t, dim=1)
    q = torch.where(ok, logq.exp(), torch.zeros_like(logq))
    loss = tau * tau * torch.where(ok & ((q > 0) | torch.isnan(q)), q * (logq - logp.gather(1, at)), torch.zeros_like(q)).sum(1)
    target = torch.zeros_like(x).scatter_add_(1, at, q)
    return loss, torch.where(is_open & live[:, None], logp.exp(), torch.zeros_like(logp)), target, is_open, live


def check_grad(grad, p, target, is_open, live, weight, tau, scale_spread):
    want = torch.where(is_open & live[:, None], weight[:, None] * tau * (p - target), torch.zeros_like(p))
    g = grad.double().cpu()
    assert g.shape == want.shape and (g[~(is_open & live[:, None])] == 0).all()
    size = (weight.abs() * tau)[:, None]
    tolerance = size * p * (LOG_Z + scale_spread * 2.0 ** -23) + size * target * 2.0 ** -24 + want.abs() * HALF_STEP[grad.dtype] + SMALLEST[grad.dtype] + size * 2.0 ** -126
    nan = torch.isnan(want)
    assert torch.equal(nan, torch.isnan(g))
    assert ((g - want).abs() <= tolerance)[~nan].all()


def check(x, ids, values, mask, tau, weight=None):
    rows, vocab = x.shape
    weight = torch.ones(rows) if weight is None else weight
    ref = reference(x, ids, values, mask, tau)
    finite = x.detach().double()[torch.isfinite(x.detach())]
    spread = float((finite.max() - finite.min()) / tau * 1.45) if finite.numel() else 0.0
    w = weight.cuda()
    leaf = x.detach().requires_grad_()
    loss = distill_loss(leaf, ids, values, mask, temperature=tau)
    again, grad2 = distill_loss_grad(x, ids, values, mask, temperature=tau, row_weight=w)
    grad, = torch.autograd.grad(loss, leaf, w)
    assert grad.shape == x.shape and grad.dtype == grad2.dtype == x.dtype and loss.dtype == again.dtype == torch.float32
    for got in (loss.detach(), again):
        got, want = got.double().cpu(), ref[0]
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        ok = ~torch.isnan(want)
        assert ((got - want).abs() <= tau * tau * LOG_Z + want.abs() * 2.0 ** -23)[ok].all()
        assert (got[~ref[4]] == 0).all()
    for g in (grad, grad2):
        check_grad(g, *ref[1:], weight.double(), tau, spread)
    return loss.detach(), grad


def make(rng, rows, vocab, k, dtype, pad=0, offset=0, teacher=torch.bfloat16, masked=True):
    x = torch.as_tensor(rng.normal(size=(rows, vocab)) * 2.5)
    buf = torch.zeros(offset + rows * (vocab + pad), dtype=dtype, device="cuda")
    view = buf[offset:].view(rows, vocab + pad)[:, :vocab]
    view.copy_(x)
    ids = torch.stack([torch.as_tensor(rng.permutation(vocab)[:k] if k <= vocab else rng.integers(vocab, size=k)) for _ in range(rows)]).int()
    values = torch.as_tensor(rng.normal(size=(rows, k)) * 2).to(teacher)
    mask = None
    if masked:
        bits = torch.as_tensor(rng.random((rows, vocab)) < rng.choice([0.97, 0.5, 0.05], size=rows)[:, None])
        if rows > 2:
            bits[2] = False                                  # nothing allowed
        mask = pack(bits).cuda()
    if rows > 3:
        ids[3] = -1                                          # nothing listed
    if rows > 4:
        ids[4, k // 2:] = -1
    if rows > 5:
        ids[5, 0] = vocab + 3                                # no token
    return view, ids.cuda(), values.cuda(), mask


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab,k,pad,offset", [(1, 1, 1, 0, 0), (3, 2, 2, 0, 0), (7, 7, 3, 1, 3), (8, 8, 8, 0, 0), (9, 9, 20, 0, 0), (33, 513, 8, 0, 0),
                                                     (12, 1003, 64, 5, 1), (6, 8192, 256, 0, 0), (6, 8200, 255, 56, 8), (9, 32000, 50, 0, 0),
                                                     (6, 100003, 65, 0, 0), (7, 128256, 64, 0, 0), (3, 163848, 1, 0, 0), (4, 200003, 128, 5, 0)])
def test_sizes_and_layouts(rows, vocab, k, pad, offset, dtype):
    rng = np.random.default_rng(BASE_SEED + vocab + rows)
    for masked, tau, teacher in ((True, 1.0, torch.bfloat16), (False, 2.0, torch.float16), (True, 0.7, torch.float32)):
        x, ids, values, mask = make(rng, rows, vocab, k, dtype, pad, offset, teacher, masked)
        check(x, ids, values, mask, tau, torch.as_tensor(rng.normal(size=rows)).float())


@pytest.mark.parametrize("dtype", DTYPES)
def test_special_values(dtype):
    """Infinities and NaNs of the student and the teacher, the type's lowest value as a mask, -inf as a mask, tokens listed twice."""
    rng = np.random.default_rng(BASE_SEED + 3)
    x, ids, values, mask = make(rng, 16, 1003, 12, dtype)
    x, low = x.clone(), torch.finfo(dtype).min
    mask[6:] = -1
    mask[:, -1] &= (1 << (1003 % 32)) - 1
    x[6, ::2] = -math.inf
    x[7] = -math.inf                                         # no open token
    x[8, ::3] = low
    x[9, 5] = math.nan
    ids[9] = torch.arange(20, 32)
    ids[10] = ids[10, 0]                                     # one token twelve times
    ids[11, 6:] = ids[11, :6]
    values[12, 3] = -math.inf
    values[13] = -math.inf                                   # no entry
    values[14, 2] = math.nan
    mask[15] = 0
    mask[15, 3] = 16                                         # one token, and the teacher lists it
    ids[15, 7] = 100
    loss, grad = check(x, ids, values, mask, 1.0)
    assert (loss[[3, 7, 13, 15]] == 0).all() and (grad[[3, 7, 13, 15]] == 0).all()
    assert torch.isnan(loss[[9, 14]]).all()
    masked = x.clone()                                       # a masked NaN or infinity is nothing
    bits = unpack(mask.cpu(), 1003).cuda()
    for junk in (math.nan, math.inf, -math.inf, low):
        masked[~bits] = junk
        other, other_grad = distill_loss_grad(masked, ids, values, mask)
        assert torch.equal(other[:9], loss[:9])
        torch.testing.assert_close(other_grad[:9], grad[:9], rtol=2 * HALF_STEP[dtype], atol=SMALLEST[dtype])


@pytest.mark.parametrize("dtype", DTYPES)
def test_large_logits_and_temperatures(dtype):
    rng = np.random.default_rng(BASE_SEED + 4)
    for scale, tau in ((100.0, 1.0), (1.0, 1 / 64), (1.0, 512.0), (3000.0, 100.0)):
        x, ids, values, mask = make(rng, 8, 1003, 9, dtype)
        x = (x.float() * scale).to(dtype)
        ref = reference(x, ids, values, mask, tau)
        spread = float((x.float().max() - x.float().min()) / tau * 1.45)
        loss, grad = distill_loss_grad(x, ids, values, mask, temperature=tau)
        # a listed token far below the top: its x is off by |x| 2^-23
        assert ((loss.double().cpu() - ref[0]).abs() <= tau * tau * (LOG_Z + spread * 2.0 ** -23) + ref[0].abs() * 2.0 ** -23).all()
        check_grad(grad, *ref[1:], torch.ones(8).double(), tau, spread)


def test_gradient_is_the_slope_of_the_loss():
    """Differences of the 64-bit loss along random directions.  With h = 1e-3 and logits in a direction of entries of size 1, the third
    derivative's share is h^2 / 6 times at most 8: 2e-6; the gradient's own errors are those above."""
    rng = np.random.default_rng(BASE_SEED + 5)
    x, ids, values, mask = make(rng, 10, 513, 16, torch.float32)
    tau, h = 1.5, 1e-3
    loss, grad = distill_loss_grad(x, ids, values, mask, temperature=tau)
    for _ in range(4):
        d = torch.as_tensor(rng.uniform(-1, 1, size=x.shape)).cuda()
        up = reference(x.double() + h * d, ids, values, mask, tau)[0]
        down = reference(x.double() - h * d, ids, values, mask, tau)[0]
        slope = (grad.double() * d).sum(1).cpu()
        assert ((up - down) / (2 * h) - slope).abs().max() <= 1e-5 + 2 * tau * LOG_Z


def test_through_autograd():
    """The upstream gradient of a mean (one number for all rows), of a part, of none; logits that are not a leaf; a second pass."""
    rng = np.random.default_rng(BASE_SEED + 6)
    x, ids, values, mask = make(rng, 12, 1003, 8, torch.bfloat16)
    _, unit = distill_loss_grad(x, ids, values, mask, temperature=2.0, row_weight=torch.full((12,), 1 / 12, device="cuda"))
    leaf = x.detach().clone().requires_grad_()
    distill_loss(leaf, ids, values, mask, temperature=2.0).mean().backward()
    assert torch.equal(leaf.grad, unit)
    hidden, head = torch.randn(12, 16, device="cuda", requires_grad=True), torch.randn(16, 1003, device="cuda", requires_grad=True)
    logits = hidden @ head
    loss = distill_loss(logits, ids, values, mask)
    (loss[:5] * 3).sum().backward(retain_graph=True)
    _, direct = distill_loss_grad(logits, ids, values, mask, row_weight=torch.tensor([3.0] * 5 + [0.0] * 7, device="cuda"))
    torch.testing.assert_close(head.grad, hidden.detach().t() @ direct, rtol=1e-5, atol=1e-5)
    before = head.grad.clone()
    (loss[:5] * 3).sum().backward()
    torch.testing.assert_close(head.grad, 2 * before)
    with torch.no_grad():
        assert torch.equal(distill_loss(logits, ids, values, mask), loss.detach())
    with pytest.raises(RuntimeError, match="differentiable once"):
        leaf = x.float().requires_grad_()
        torch.autograd.grad(distill_loss(leaf, ids, values, mask).sum(), leaf, create_graph=True)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [1003, 100003])
def test_gradient_in_place_of_the_logits(vocab, dtype):
    rng = np.random.default_rng(BASE_SEED + 7)
    x, ids, values, mask = make(rng, 9, vocab, 30, dtype, pad=3)
    loss, grad = distill_loss_grad(x, ids, values, mask)
    again, same = distill_loss_grad(x, ids, values, mask, out=x)
    assert same is x and torch.equal(x, grad) and torch.equal(loss, again)
    wide = torch.full((9, vocab + 9), 5.0, dtype=dtype, device="cuda")
    x, ids, values, mask = make(rng, 9, vocab, 30, dtype)
    _, apart = distill_loss_grad(x, ids, values, mask)
    distill_loss_grad(x, ids, values, mask, out=wide[:, 2:vocab + 2])
    assert torch.equal(wide[:, 2:vocab + 2], apart) and (wide[:, :2] == 5).all() and (wide[:, vocab + 2:] == 5).all()


def test_a_list_of_one_is_the_cross_entropy():
    rng = np.random.default_rng(BASE_SEED + 8)
    x, ids, values, mask = make(rng, 20, 513, 1, torch.float32)
    ids = torch.as_tensor(rng.integers(513, size=(20, 1))).int().cuda()
    mask[torch.arange(20), ids[:, 0].long() // 32] |= (1 << (ids[:, 0] % 32)).int()
    loss, grad = check(x, ids, values, mask, 1.0)
    y = torch.where(unpack(mask.cpu(), 513), x.double().cpu(), torch.full(x.shape, -math.inf, dtype=torch.float64))
    want = torch.nn.functional.cross_entropy(y, ids[:, 0].long().cpu(), reduction="none")
    assert (loss.double().cpu() - want).abs().max() <= LOG_Z


def test_the_teachers_list_of_the_top_k_call():
    """Rows that apply_mask_topk pads are taken as they are."""
    rng = np.random.default_rng(BASE_SEED + 9)
    rows, vocab, k = 11, 32000, 32
    text = np.append(np.resize(np.frombuffer(b"a+*()", dtype=np.uint8), vocab - 1), np.uint8(0))
    lib = Pre3(G.ARITHMETIC, text, np.append(np.arange(vocab), vocab - 1), vocab - 1, stack_cap=8)
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    lib.bind_state(i32(rows), i32(rows, 8), i32(rows) + 1, i32(rows))
    x, _, _, mask = make(rng, rows, vocab, k, torch.bfloat16)
    mask[1] = 0
    mask[1, 7] = 0b1011
    teacher = (x.float() + torch.randn_like(x.float())).bfloat16()
    ids, values = i32(rows, k), torch.zeros((rows, k), dtype=torch.bfloat16, device="cuda")
    lib.apply_mask_topk(teacher, mask, ids, values)
    assert (ids[1, 3:] == -1).all() and (ids[2] == -1).all()
    check(x, ids, values, mask, 2.0)


def test_in_a_graph_and_on_another_stream():
    rng = np.random.default_rng(BASE_SEED + 10)
    x, ids, values, mask = make(rng, 24, 32000, 20, torch.bfloat16)
    weight, out = torch.rand(24, device="cuda"), torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        distill_loss_grad(x, ids, values, mask, row_weight=weight, out=out)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss, _ = distill_loss_grad(x, ids, values, mask, row_weight=weight, out=out)
    for _ in range(4):
        x.normal_()
        weight.uniform_()
        graph.replay()
        got, got_grad = loss.clone(), out.clone()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            want, want_grad = distill_loss_grad(x, ids, values, mask, row_weight=weight)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(got_grad, want_grad)


def test_rows_beyond_32_bit_offsets():
    """40,000 rows of 70,016 logits in 16 bits: the last ones lie beyond 2^32 bytes and 2^31 elements."""
    rows, vocab, k = 40000, 70016, 4
    x = torch.empty((rows, vocab), dtype=torch.float16, device="cuda").normal_()
    ids = torch.full((rows, k), -1, dtype=torch.int32, device="cuda")
    ids[-3:] = torch.randint(vocab, (3, k), device="cuda", dtype=torch.int32)
    values = torch.randn((rows, k), device="cuda")
    loss, grad = distill_loss_grad(x, ids, values, None)
    assert (loss[:-3] == 0).all() and not grad[:-3].any()
    ref = reference(x[-3:], ids[-3:], values[-3:], None, 1.0)
    assert ((loss[-3:].double().cpu() - ref[0]).abs() <= LOG_Z + ref[0].abs() * 2.0 ** -23).all()
    check_grad(grad[-3:], *ref[1:], torch.ones(3).double(), 1.0, 16.0)
    check(x[-3:], ids[-3:].contiguous(), values[-3:].contiguous(), None, 1.0)


def test_an_empty_batch():
    x = torch.empty((0, 513), dtype=torch.bfloat16, device="cuda", requires_grad=True)
    ids, values = torch.empty((0, 4), dtype=torch.int32, device="cuda"), torch.empty((0, 4), device="cuda")
    loss = distill_loss(x, ids, values)
    loss.sum().backward()
    assert loss.shape == (0,) and x.grad.shape == (0, 513)
    assert distill_loss_grad(x, ids, values)[1].shape == (0, 513)


@pytest.mark.parametrize("rows,vocab", [(65536, 9), (70001, 40)])
def test_more_rows_than_a_grids_other_dimensions_have(rows, vocab):
    rng = np.random.default_rng(BASE_SEED + 11)
    x = torch.as_tensor(rng.normal(size=(rows, vocab))).bfloat16().cuda()
    ids = torch.as_tensor(rng.integers(-1, vocab, size=(rows, 2))).int().cuda()
    values = torch.as_tensor(rng.normal(size=(rows, 2))).float().cuda()
    check(x, ids, values, None, 1.5, torch.as_tensor(rng.normal(size=rows)).float())


@pytest.mark.parametrize("rows,vocab,dtype", [(1535, 2000, torch.bfloat16), (1536, 2000, torch.bfloat16), (1536, 6144, torch.float32), (1536, 6145, torch.float32),
                                              (3, 16384, torch.float32), (3, 16385, torch.float32), (3, 24575, torch.float16), (160, 24576, torch.bfloat16),
                                              (161, 24576, torch.bfloat16), (3, 28001, torch.bfloat16), (770, 28001, torch.bfloat16), (3, 36864, torch.bfloat16),
                                              (3, 36865, torch.bfloat16), (170, 56001, torch.float16)])
def test_sizes_at_the_lines_between_forms(rows, vocab, dtype):
    """Threads of a block and blocks of a row, both sides of where they change."""
    gen = torch.Generator(device="cuda").manual_seed(BASE_SEED + rows + vocab)
    x = (3 * torch.randn((rows, vocab), generator=gen, device="cuda")).to(dtype)
    ids = torch.randint(-1, vocab, (rows, 12), generator=gen, device="cuda", dtype=torch.int32)
    values = torch.randn((rows, 12), generator=gen, device="cuda").bfloat16()
    mask = pack(torch.rand((rows, vocab), generator=torch.Generator().manual_seed(BASE_SEED + vocab)) < 0.7).cuda()
    check(x, ids, values, mask, 1.5)


@pytest.mark.parametrize("rows,vocab,dtype", [(161, 80000, torch.bfloat16), (161, 80001, torch.bfloat16), (200, 100003, torch.float16), (256, 28001, torch.float32),
                                              (257, 28001, torch.float32), (257, 56001, torch.float32), (769, 28001, torch.float16)])
def test_sizes_at_the_lines_of_the_longest_rows(rows, vocab, dtype):
    test_sizes_at_the_lines_between_forms(rows, vocab, dtype)


@pytest.mark.parametrize("rows,vocab", [(200, 20011), (200, 128256), (257, 128256)])
def test_a_mass_of_small_weights_beside_a_large_one(rows, vocab):
    """One token of weight 1 and a vocabulary of weight 5.5e-8 each, less than half a step of 1 in 32 bits.  A weight of the mass is off by
    less than (2 * 24 * 0.7 + 2 + 16 + 3 * 36) 2^-24 < 2^-16 of itself (exponent, exponential, a sum of sixteen, three joins of threads), the
    mass is 0.0071 at most, and the token of weight 1 is exact: the loss, log Z, is off by less than 2^-22."""
    x = torch.full((rows, vocab), -16.72, device="cuda")
    at = torch.arange(rows, device="cuda") % 64 * 8
    x[torch.arange(rows, device="cuda"), at] = 0.0
    ids, values = at[:, None].int().contiguous(), torch.zeros((rows, 1), device="cuda")
    want = math.log1p((vocab - 1) * math.exp(float(x[0, 1]) - float(x[0, 0])))
    loss, grad = distill_loss_grad(x, ids, values)
    assert (loss.double() - want).abs().max() <= 2.0 ** -22
    assert (distill_loss(x, ids, values).double() - want).abs().max() <= 2.0 ** -22
    p = -math.expm1(-want)                                   # of the mass
    assert (grad[torch.arange(rows, device="cuda"), at].double() + p).abs().max() <= 2.0 ** -22
