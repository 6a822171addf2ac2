"""The cross entropy of a head, its gradients, against the definition in 64 bits.

What may be off, by arithmetic.  With u = 2^-24 (32-bit sums) and r half a step of the operands' type (bf16 2^-8, f16 2^-11; 32-bit operands and slopes are
sums of three bf16 numbers, to 2^-24, whose left-out products are 4 of 2^-24 at most):
  a logit      e = (dim + 16) * u * sum |h w|, for 32-bit operands 8 u * sum |h w| more and six times as many sums
  the loss     two such logits' errors (the target's, and the sum's, whose weights are a mean), the exponentials' and their sums' 2^-16, and a rounding
  a slope      |g| (p (2 e + 2^-16) + (r + 2^-20) |p - [t]|), and for f16 half a step of the smallest numbers, 2^-25, in units of 2^-14 max |g| / 2
  a gradient   the slopes' errors times what they are multiplied with, (number of terms + 16) * u (f32: 6 times that, and 8 u) of the sum of the products'
               absolute values, half a step of the result
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
U = 2.0 ** -24


def pack(bits):
    rows, vocab = bits.shape
    x = torch.zeros((rows, -(-vocab // 32) * 32), dtype=torch.int64, device=bits.device)
    x[:, :vocab] = bits
    x = (x.view(rows, -1, 32) << torch.arange(32, device=bits.device)).sum(dim=2)
    return torch.where(x >= 2 ** 31, x - 2 ** 32, x).int().contiguous()


def inputs(dtype, rows, vocab, dim, mask=None, seed=0, strided=False, ids=torch.int32):
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def laid(x):
        if not strided:
            return x.to(TYPES[dtype])
        room = torch.full((x.shape[0], x.shape[1] + 5), math.nan, dtype=TYPES[dtype], device="cuda")
        room[:, 3:3 + x.shape[1]] = x
        return room[:, 3:3 + x.shape[1]]

    weight = laid(normal(vocab, dim) * (2 / math.sqrt(dim)))
    targets = torch.randint(vocab, (rows,), generator=gen, device="cuda")
    hidden = laid(normal(rows, dim) + 1.5 * weight.float()[targets])
    if rows > 2:                                                    # rows that teach nothing
        targets[::5] = torch.tensor([-1, -100, vocab, 2 ** 31 - 1, -2 ** 31], device="cuda")[torch.arange(len(targets[::5]), device="cuda") % 5]
    allowed = None
    if mask is not None:
        share = torch.tensor([0.95, 0.5, 3 / vocab, 0.0], device="cuda")[torch.arange(rows, device="cuda") % 4] if mask == "mixed" else torch.full((rows,), mask, device="cuda")
        allowed = torch.rand((rows, vocab), generator=gen, device="cuda") < share[:, None]
        inside = (targets >= 0) & (targets < vocab) & (torch.arange(rows, device="cuda") % 7 != 3)
        allowed[torch.nonzero(inside)[:, 0], targets[inside]] = True
    weights = torch.rand(rows, generator=gen, device="cuda") + 0.5
    return hidden, weight, targets.to(ids), allowed, weights


def reference(hidden, weight, targets, allowed, g, dtype):
    """Losses and gradients in 64 bits, and how far off each may be."""
    h, w, t = hidden.double(), weight.double(), targets.long()
    rows, vocab, dim = len(h), len(w), w.shape[1]
    r = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}[dtype]
    many, extra = (6, 8 * U) if dtype == "f32" else (1, 0.0)
    inside = (t >= 0) & (t < vocab)
    t = t.clamp(0, vocab - 1)
    if allowed is not None:
        inside = inside & allowed[torch.arange(rows, device="cuda"), t]
    taught = torch.nonzero(inside)[:, 0]
    h_t, t, g_t = h[taught], t[taught], g.double()[taught]
    open_ = torch.ones((len(taught), vocab), dtype=torch.bool, device="cuda") if allowed is None else allowed[taught]
    x = h_t @ w.T
    size = h_t.abs() @ w.abs().T
    e = ((many * dim + 16) * U + extra) * size.masked_fill(~open_, 0).amax(dim=1, keepdim=True)
    x = x.masked_fill(~open_, -math.inf)
    logp = torch.log_softmax(x, dim=1)
    loss, off_loss = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda")
    at = torch.arange(len(taught), device="cuda")
    loss[taught] = -logp[at, t]
    off_loss[taught] = 2 * e[:, 0] + 2.0 ** -16 + 2.0 ** -23 * loss[taught].abs()
    p = torch.exp(logp)
    one = torch.zeros_like(p)
    one[at, t] = 1
    s = (p - one) * g_t[:, None]
    off_s = g_t[:, None].abs() * (p * (2 * e + 2.0 ** -16) + (r + 2.0 ** -20) * (p - one).abs())
    if dtype == "f16" and len(taught):
        off_s = off_s + 2.0 ** -25 * 2.0 ** -13 * g_t.abs().max() * open_
    d_h, off_h = torch.zeros_like(h), torch.zeros_like(h)
    d_h[taught] = s @ w
    off_h[taught] = off_s @ w.abs() + ((many * vocab + 16) * U + extra) * (s.abs() @ w.abs())
    d_w = s.T @ h_t
    off_w = off_s.T @ h_t.abs() + ((many * len(taught) + 16) * U + extra) * (s.abs().T @ h_t.abs())
    half = torch.finfo(TYPES[dtype]).eps / 2
    tiny = torch.finfo(TYPES[dtype]).tiny
    return (loss, off_loss), (d_h, off_h * (1 + half) + half * d_h.abs() + tiny * 2.0 ** -8), (d_w, off_w * (1 + half) + half * d_w.abs() + tiny * 2.0 ** -8)


def close(got, want, what):
    exact, off = want
    assert not torch.isnan(got).any(), what
    bad = (got.double() - exact).abs() > off
    assert not bad.any(), (what, int(bad.sum()), float(((got.double() - exact).abs() / off.clamp(min=1e-300)).max()))


CASES = [
    # dtype, rows, vocab, dim, mask, strided
    ("bf16", 8, 3001, 520, "mixed", False), ("f16", 7, 700, 1001, "mixed", True), ("f32", 8, 1003, 130, 0.5, False), ("f32", 2, 40000, 24, None, False),
    ("bf16", 9, 20000, 256, "mixed", False), ("f32", 791, 145, 1000, None, False), ("bf16", 400, 60, 2000, "mixed", False), ("f16", 33, 30001, 130, 0.5, False),
    ("bf16", 1, 1, 1, None, False), ("f32", 1, 1, 1, None, False), ("f16", 2, 31, 7, None, False),
    ("bf16", 1, 5000, 512, None, False), ("bf16", 33, 513, 64, "mixed", False), ("bf16", 64, 1025, 200, "mixed", True),
    ("bf16", 65, 257, 72, 0.5, False), ("bf16", 129, 2000, 100, "mixed", False), ("bf16", 300, 4097, 136, "mixed", False),
    ("bf16", 515, 1100, 320, None, True), ("f16", 5, 513, 64, "mixed", False), ("f16", 100, 3001, 1001, None, False), ("f16", 257, 700, 48, "mixed", True),
    ("f32", 3, 513, 512, "mixed", False), ("f32", 64, 513, 100, "mixed", False), ("f32", 130, 1003, 65, None, True), ("f32", 260, 600, 128, "mixed", False),
]


@pytest.mark.parametrize("dtype,rows,vocab,dim,mask,strided", CASES)
def test_loss_and_gradients(dtype, rows, vocab, dim, mask, strided):
    from paper_2506_03887_amd import head_loss, head_loss_grad
    hidden, weight, targets, allowed, g = inputs(dtype, rows, vocab, dim, mask, seed=rows + vocab, strided=strided, ids=torch.int64 if rows % 2 else torch.int32)
    if rows <= 2:
        targets[0] = vocab - 1
    bits = None if allowed is None else pack(allowed)
    want = reference(hidden, weight, targets, allowed, g, dtype)
    print(f"[head] {dtype} {rows} x {vocab} x {dim} mask {mask} strided {strided}", flush=True)
    close(head_loss(hidden, weight, targets, bits), want[0], "loss")
    got = head_loss_grad(hidden, weight, targets, bits, row_weight=g)
    for x, y, what in zip(got, want, ("loss", "hidden", "weight")):
        close(x, y, what)
    h, w = hidden.detach().requires_grad_(), weight.detach().requires_grad_()
    loss = head_loss(h, w, targets, bits)
    by_autograd = torch.autograd.grad(loss, (h, w), g)
    assert torch.equal(loss.detach(), got[0])
    for a, b in zip(by_autograd, got[1:]):
        assert torch.equal(a, b)                                    # one path, in one order
    h_only, = torch.autograd.grad(head_loss(h, weight, targets, bits), (h,), g)
    w_only, = torch.autograd.grad(head_loss(hidden, w, targets, bits), (w,), g)
    assert torch.equal(h_only, got[1]) and torch.equal(w_only, got[2])


@pytest.mark.parametrize("dtype,rows,vocab,dim,mask,strided", [("f32", 9, 9000, 130, "mixed", False), ("f32", 33, 2100, 513, "mixed", True), ("f32", 64, 4097, 257, None, True),
                                                               ("f32", 17, 301, 5003, 0.5, False), ("f16", 20, 70001, 1001, "mixed", False), ("bf16", 50, 520000, 130, None, True)])
def test_a_loss_alone_of_weights_as_they_lie(dtype, rows, vocab, dim, mask, strided):
    from paper_2506_03887_amd import head_loss
    hidden, weight, targets, allowed, g = inputs(dtype, rows, vocab, dim, mask, seed=rows, strided=strided)
    want = reference(hidden, weight, targets, allowed, g, dtype)[0]
    print(f"[head] {dtype} {rows} x {vocab} x {dim} mask {mask} strided {strided}", flush=True)
    close(head_loss(hidden, weight, targets, None if allowed is None else pack(allowed)), want, "loss")


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_vocabulary_in_pieces(dtype):
    """Several pieces' slopes and sums: what a piece takes is held below a gigabyte."""
    from paper_2506_03887_amd import head_loss_grad
    rows, vocab, dim = (4000, 70001, 64) if dtype != "f32" else (2000, 45001, 40)
    hidden, weight, targets, allowed, g = inputs(dtype, rows, vocab, dim, None, seed=3)
    want = reference(hidden, weight, targets, allowed, g, dtype)
    for x, y, what in zip(head_loss_grad(hidden, weight, targets, None, row_weight=g), want, ("loss", "hidden", "weight")):
        close(x, y, what)


def test_no_row_teaches():
    from paper_2506_03887_amd import head_loss_grad
    hidden, weight, targets, _, _ = inputs("bf16", 40, 300, 64)
    hidden[:] = math.nan
    for case, mask in ((torch.full_like(targets, -1), None), (targets.clamp(0, 299), torch.zeros((40, 10), dtype=torch.int32, device="cuda"))):
        loss, d_h, d_w = head_loss_grad(hidden, weight, case, mask)
        assert not loss.any() and not d_h.any() and not d_w.any()
    loss, d_h, d_w = head_loss_grad(hidden[:0], weight, targets[:0])
    assert loss.shape == (0,) and d_h.shape == (0, 64) and d_w.shape == weight.shape and not d_w.any()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_what_is_not_taught_or_not_allowed_may_hold_anything(dtype):
    """NaNs and infinities in rows without a target, and in the weights of tokens that no row allows, reach nothing."""
    from paper_2506_03887_amd import head_loss_grad
    hidden, weight, targets, allowed, g = inputs(dtype, 70, 600, 96, "mixed", seed=5)
    nowhere = ~allowed[:, 100:140].any(dim=1).all()
    allowed[:, 100:140] = False
    bits = pack(allowed)
    good = head_loss_grad(hidden, weight, targets, bits, row_weight=g)
    t = targets.long()
    taught = (t >= 0) & (t < 600)
    taught[taught.clone()] &= allowed[torch.nonzero(taught)[:, 0], t[taught]]
    h, w, g2 = hidden.clone(), weight.clone(), g.clone()
    h[~taught] = math.nan
    h[~taught, ::3] = math.inf
    g2[~taught] = math.nan
    w[100:140] = math.nan
    w[110:120] = -math.inf
    w[120:130] = math.inf
    for a, b in zip(head_loss_grad(h, w, targets, bits, row_weight=g2), good):
        assert torch.equal(a, b)
    del nowhere


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows,vocab,dim", [(5, 3000, 96), (40, 3000, 200), (300, 1000, 96), (900, 20000, 512)])
def test_numbers_behind_the_mask(dtype, rows, vocab, dim):
    """NaNs and infinities in the weights of tokens that no row allows, in a graph whose replays have them and do not: results as without."""
    from paper_2506_03887_amd import head_loss_grad
    hidden, weight, targets, allowed, g = inputs(dtype, rows, vocab, dim, 0.5, seed=7)
    allowed[:, 10:13] = False
    allowed[:, vocab - 3:] = False
    targets[(targets >= 10) & (targets < 13)] = 0
    bits = pack(allowed)
    good = [x.clone() for x in head_loss_grad(hidden, weight, targets, bits, row_weight=g)]
    clean, wild = weight.clone(), weight.clone()
    wild[10], wild[11, ::2], wild[12, dim // 2] = math.nan, math.inf, -math.inf
    wild[vocab - 1, 0], wild[vocab - 2] = math.nan, -math.inf
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = head_loss_grad(hidden, weight, targets, bits, row_weight=g)
    for numbers in (wild, clean, wild, clean):
        weight.copy_(numbers)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, good):
            assert torch.equal(a, b)
    eager = head_loss_grad(hidden, wild, targets, bits, row_weight=g)
    assert all(torch.equal(a, b) for a, b in zip(eager, good))


@pytest.mark.parametrize("rows,vocab,dim", [(5, 3000, 96), (40, 3000, 200), (300, 20000, 512)])
def test_a_row_of_nans_leaves_the_others(rows, vocab, dim):
    """A row that allows a weight which is NaN, and rows that do not: their gradients are theirs."""
    from paper_2506_03887_amd import head_loss_grad
    hidden, weight, targets, allowed, g = inputs("bf16", rows, vocab, dim, 0.5, seed=8)
    targets[:] = torch.randint(100, vocab, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    allowed[torch.arange(rows, device="cuda"), targets.long()] = True
    allowed[:, 40:42] = False
    loss, d_h, _ = head_loss_grad(hidden, weight, targets, pack(allowed), row_weight=g)
    weight[40], weight[41, 3] = math.nan, math.inf
    allowed[1, 40], allowed[2, 41] = True, True
    hidden[2, 3] = -1.0                                             # (a logit of -inf: the token has no share; its slope is 0, times inf NaN at one place)
    hidden_of = torch.arange(rows, device="cuda")
    other = (hidden_of != 1) & (hidden_of != 2)
    loss2, d_h2, d_w2 = head_loss_grad(hidden, weight, targets, pack(allowed), row_weight=g)
    assert torch.equal(loss2[other], loss[other]) and torch.equal(d_h2[other], d_h[other])
    assert torch.isnan(loss2[1]) and torch.isnan(d_h2[1]).all() and torch.isfinite(loss2[2])
    assert torch.isnan(d_w2[40]).all()


def test_nans_come_out():
    from paper_2506_03887_amd import head_loss_grad
    hidden, weight, targets, _, g = inputs("bf16", 9, 400, 64, seed=6)
    targets = torch.arange(9, dtype=torch.int32, device="cuda")
    hidden[4, 7] = math.nan
    loss, d_h, d_w = head_loss_grad(hidden, weight, targets)
    assert torch.isnan(loss).nonzero()[:, 0].tolist() == [4] and torch.isnan(d_h).any(dim=1).nonzero()[:, 0].tolist() == [4] and torch.isnan(d_w).all()


def test_gradient_by_differences():
    """The gradient of 32-bit operands against differences of 64-bit losses along random directions."""
    from paper_2506_03887_amd import head_loss_grad
    hidden, weight, targets, allowed, g = inputs("f32", 40, 300, 50, "mixed", seed=8)
    loss, d_h, d_w = head_loss_grad(hidden, weight, targets, pack(allowed), row_weight=g)
    t = targets.long()
    taught = (t >= 0) & (t < 300)
    taught[taught.clone()] &= allowed[torch.nonzero(taught)[:, 0], t[taught]]

    def total(h, w):
        x = (h @ w.T).masked_fill(~allowed, -math.inf)[taught]
        return (torch.nn.functional.cross_entropy(x, t[taught], reduction="none") * g.double()[taught]).sum()

    gen = torch.Generator(device="cuda").manual_seed(9)
    for _ in range(4):
        a, b = (torch.randn(x.shape, generator=gen, device="cuda", dtype=torch.float64) for x in (hidden, weight))
        step = 1e-4                                                 # the error of a central difference: about step^2 of the third derivative
        along = (total(hidden.double() + step * a, weight.double() + step * b) - total(hidden.double() - step * a, weight.double() - step * b)) / (2 * step)
        got = (d_h.double() * a).sum() + (d_w.double() * b).sum()
        assert abs(float(got - along)) <= 1e-4 * float((d_h.abs().double() * a.abs()).sum() + (d_w.abs().double() * b.abs()).sum())


def test_small_weights_of_f16_rows():
    """Weights as a mean over a large batch has them, times a small loss scale: slopes below what f16 holds by itself."""
    from paper_2506_03887_amd import head_loss_grad
    hidden, weight, targets, allowed, g = inputs("f16", 100, 800, 64, "mixed", seed=10)
    bits = pack(allowed)
    _, d_h, d_w = head_loss_grad(hidden, weight, targets, bits, row_weight=g * 2.0 ** 6)
    _, e_h, e_w = head_loss_grad(hidden, weight, targets, bits, row_weight=g * 2.0 ** -6)
    some = e_w.abs() > 2.0 ** -13                                   # (normal numbers: the power of two passes through unrounded)
    assert some.any() and torch.equal(e_w[some].float() * 2.0 ** 12, d_w[some].float())


def test_a_captured_step_replayed():
    """Loss and gradients in a graph, replayed on new inputs with eager work in between, against the eager call."""
    from paper_2506_03887_amd import head_loss_grad
    one = inputs("bf16", 100, 3000, 128, "mixed", seed=11)
    two = inputs("bf16", 100, 3000, 128, "mixed", seed=12)
    hidden, weight, targets, g = (x.clone() for x in (one[0], one[1], one[2], one[4]))
    bits = pack(one[3])
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        head_loss_grad(hidden, weight, targets, bits, row_weight=g)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = head_loss_grad(hidden, weight, targets, bits, row_weight=g)
    for turn in range(4):
        h, w, t, allowed, k = (one, two)[turn % 2]
        for to, x in ((hidden, h), (weight, w), (targets, t), (g, k), (bits, pack(allowed))):
            to.copy_(x)
        graph.replay()
        want = head_loss_grad(h, w, t, pack(allowed), row_weight=k)
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b), turn


def test_on_another_stream_and_twice_at_once():
    from paper_2506_03887_amd import head_loss_grad
    cases = [inputs("bf16", 200, 2000, 256, "mixed", seed=s) for s in (13, 14)]
    want = [head_loss_grad(c[0], c[1], c[2], pack(c[3]), row_weight=c[4]) for c in cases]
    masks = [pack(c[3]) for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    got = []
    for c, m, s in zip(cases, masks, streams):
        with torch.cuda.stream(s):
            got.append([head_loss_grad(c[0], c[1], c[2], m, row_weight=c[4]) for _ in range(3)])
    torch.cuda.synchronize()
    for results, w in zip(got, want):
        for r in results:
            assert all(torch.equal(a, b) for a, b in zip(r, w))


def test_a_scalar_loss_and_broadcast_gradients():
    """mean().backward(): the rows' gradients are one number, repeated without memory of its own."""
    from paper_2506_03887_amd import head_loss, head_loss_grad
    hidden, weight, targets, _, _ = inputs("bf16", 50, 400, 64, seed=15)
    h, w = hidden.requires_grad_(), weight.requires_grad_()
    head_loss(h, w, targets).mean().backward()
    _, d_h, d_w = head_loss_grad(hidden, weight, targets, row_weight=torch.full((50,), 1 / 50, device="cuda"))
    assert torch.equal(h.grad, d_h) and torch.equal(w.grad, d_w)


def test_inputs_overwritten_before_the_backward_pass():
    from paper_2506_03887_amd import head_loss
    hidden, weight, targets, _, _ = inputs("bf16", 20, 100, 64, seed=16)
    loss = head_loss(hidden.requires_grad_(), weight, targets)
    weight += 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.sum().backward()


def test_a_second_derivative_is_refused():
    from paper_2506_03887_amd import head_loss
    hidden, weight, targets, _, _ = inputs("f32", 5, 40, 8, seed=17)
    with pytest.raises(RuntimeError, match="differentiable once"):
        torch.autograd.grad(head_loss(hidden.requires_grad_(), weight, targets).sum(), hidden, create_graph=True)


@pytest.mark.parametrize("dtype,rows,vocab,dim", [("bf16", 5, 1003, 72), ("f16", 40, 1003, 77), ("f32", 300, 700, 33), ("bf16", 700, 9000, 200)])
def test_strided_gradients_and_kept_logits_at_the_c_abi(dtype, rows, vocab, dim):
    """Gradients in rows of any stride and alignment, nothing written beside them; the gradients alone, with what the loss's call has kept and without."""
    import ctypes as c

    from paper_2506_03887_amd import head_loss_grad
    from test_matrices_arguments import Head, lib
    hidden, weight, targets, allowed, g = inputs(dtype, rows, vocab, dim, "mixed", seed=21, strided=True)
    bits = pack(allowed)
    want = head_loss_grad(hidden, weight, targets, bits, row_weight=g)
    kind = {"bf16": 0, "f16": 1, "f32": 2}[dtype]
    h = Head(hidden.data_ptr(), weight.data_ptr(), targets.data_ptr(), bits.data_ptr(), hidden.stride(0), weight.stride(0), kind, 4, rows, vocab, dim)
    of = lib()
    need, keep = of.pre3_head_workspace_bytes(c.byref(h), 1), of.pre3_head_kept_bytes(c.byref(h))
    workspace = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    kept = torch.empty(keep + 16, dtype=torch.uint8, device="cuda")
    h.workspace, h.workspace_bytes = (workspace.data_ptr() + 255) // 256 * 256, need
    stream = torch.cuda.current_stream().cuda_stream
    for has in (True, False):
        h.kept = kept.data_ptr() if has and keep else None
        loss, stats = torch.full((rows,), 9.0, device="cuda"), torch.empty((rows, 2), device="cuda")
        rooms = [torch.full((n + 1, dim + 7), 5.0, dtype=TYPES[dtype], device="cuda") for n in (rows, vocab)]
        d_h, d_w = (x[:-1, 3:3 + dim] for x in rooms)
        assert of.pre3_head_loss(c.byref(h), loss.data_ptr(), stats.data_ptr(), stream) == 0
        workspace.fill_(255)                                        # (a workspace holds nothing between calls)
        assert of.pre3_head_grad(c.byref(h), stats.data_ptr(), g.data_ptr(), 1, d_h.data_ptr(), dim + 7, d_w.data_ptr(), dim + 7, stream) == 0
        assert torch.equal(loss, want[0]) and torch.equal(d_h, want[1]) and torch.equal(d_w, want[2])
        for x in rooms:
            assert (x[-1] == 5).all() and (x[:, :3] == 5).all() and (x[:, 3 + dim:] == 5).all()


def test_a_graph_kept_for_two_backward_passes():
    from paper_2506_03887_amd import head_loss
    for rows in (6, 40, 200):
        hidden, weight, targets, allowed, g = inputs("bf16", rows, 900, 64, "mixed", seed=22)
        h, w = hidden.requires_grad_(), weight.requires_grad_()
        loss = head_loss(h, w, targets, pack(allowed))
        first = torch.autograd.grad(loss, (h, w), g, retain_graph=True)
        again = torch.autograd.grad(loss, (h, w), g)
        assert all(torch.equal(a, b) for a, b in zip(first, again))
