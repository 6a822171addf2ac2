"""What is measured of the operators on a vocabulary under a token mask: the sampler that a decode step ends with, and the loss
that teaches a small model the answers of a large one.

  sample    one token a row from [rows, vocab] logits behind the mask, by temperature, top-k, top-p and min-p, from one given random
            number a row; the token, its log-probability in what was drawn from, and how many tokens that were
  distill   the loss of a student's logits against a teacher's k best logits (what apply_mask_topk lists), both under the mask, and the
            gradient of the weighted rows: through autograd ("step"), or loss and gradient in one pass ("pass")

The order of the draw is that of the logits, descending, equal ones by ascending id; every filter keeps a prefix of it.

A case names
  op        sample | distill
  form      of distill: step | pass
  dtype     of the logits (and of the gradient): bf16 | f16 | f32
  rows, vocab, stride (elements from row to row)
  mask      none | text (rows inside a string allow nearly everything, others a number's or a structure's tokens) | schema (a
            handful of tokens in most rows)
  filters   of sample: none | top_k | top_p | min_p | mixed (all of them, each row its own values, some rows greedy)
  k         of distill: the teacher's tokens a row
  tau       of distill: the temperature of both distributions
"""
import functools
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _sample(name, dtype, rows, vocab, mask, filters, stride=None):
    case = dict(op="sample", dtype=dtype, rows=rows, vocab=vocab, stride=stride or vocab, mask=mask, filters=filters)
    return dict(case, name=name) if name else case


def _distill(name, form, dtype, rows, vocab, mask, k, tau, stride=None):
    case = dict(op="distill", form=form, dtype=dtype, rows=rows, vocab=vocab, stride=stride or vocab, mask=mask, k=k, tau=tau)
    return dict(case, name=name) if name else case


def listed():
    return [
        # the smallest call: four sequences and a vocabulary of odd size, every filter, logits in 32 bits
        _sample("sample 4 small f32", "f32", 4, 513, "text", "mixed"),
        # one user's document: the latency of a nucleus draw
        _sample("sample 1 top-p", "bf16", 1, 128256, "text", "top_p"),
        # a small server
        _sample("sample 64 top-k", "bf16", 64, 32000, "text", "top_k"),
        # the common serving batch, each request with parameters of its own
        _sample("sample 256 mixed", "bf16", 256, 128256, "text", "mixed"),
        # structured output of a fixed schema, a large batch and vocabulary
        _sample("sample 512 min-p", "bf16", 512, 152064, "schema", "min_p"),
        # free text in 16-bit floats: no grammar, nothing cut, rows off 16-byte boundaries
        _sample("sample 96 plain f16", "f16", 96, 100003, "none", "none"),
        # a model that hands out its logits in 32 bits
        _sample("sample 128 top-p f32", "f32", 128, 128256, "text", "top_p"),
        # a toy student: launches and latency
        _distill("distill step 64 small f32", "step", "f32", 64, 513, "text", 8, 1.0),
        # one long answer, odd rows
        _distill("distill step 96 f16", "step", "f16", 96, 100003, "none", 50, 2.0),
        # a batch of answers, the loss one term of several: through autograd
        _distill("distill step 2048", "step", "bf16", 2048, 32000, "text", 20, 2.0),
        # logits in 32 bits, loss and gradient at once
        _distill("distill pass 256 f32", "pass", "f32", 256, 128256, "text", 64, 1.0),
        # the largest: a training step's logits of eight answers of 512 tokens
        _distill("distill pass 4096", "pass", "bf16", 4096, 128256, "text", 64, 2.0),
    ]


def _spread(rng, lo, hi):
    """An integer of lo..hi, spread over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    vocab = _spread(rng, 100, 200_000)
    stride = rng.choice((vocab, vocab, -(-vocab // 64) * 64, -(-vocab // 8) * 8))
    dtype, mask = rng.choice(("bf16", "bf16", "f16", "f32")), rng.choice(("none", "text", "text", "schema"))
    if rng.random() < 0.55:
        rows = _spread(rng, 1, min(1024, 512 * 152064 // vocab))
        return _sample(None, dtype, rows, vocab, mask, rng.choice(("none", "top_k", "top_p", "min_p", "mixed")), stride)
    rows = _spread(rng, 8, min(8192, (2048 if dtype == "f32" else 4096) * 128256 // vocab))
    return _distill(None, rng.choice(("step", "pass")), dtype, rows, vocab, mask, rng.randint(1, min(vocab, 128)), rng.choice((1.0, 1.5, 2.0, 4.0)), stride)


# ------------------------------------------------------------------------------------------------- inputs

def _pack(bits):
    """[rows, vocab] truth values -> [rows, ceil(vocab / 32)] int32 words, least significant bit first."""
    rows, vocab = bits.shape
    words = -(-vocab // 32)
    x = torch.zeros((rows, words * 32), dtype=torch.int32, device=bits.device)
    x[:, :vocab] = bits
    x = x.view(rows, words, 32) << torch.arange(32, dtype=torch.int32, device=bits.device)
    return x.sum(dim=2, dtype=torch.int32)


def _unpack(words, vocab):
    bits = (words.unsqueeze(2) >> torch.arange(32, dtype=torch.int32, device=words.device)) & 1
    return bits.reshape(words.shape[0], -1)[:, :vocab].to(torch.bool)


def _mask(kind, rows, vocab, gen, dev):
    if kind == "none":
        return None
    # the share of the vocabulary that a row allows: nearly all of it within a string, a number's tokens, a structure's
    pick = torch.rand(rows, generator=gen, device=dev)
    few = (3 + 60 * torch.rand(rows, generator=gen, device=dev)) / vocab
    dense, numbers = (0.7, 0.85) if kind == "text" else (0.15, 0.25)
    share = torch.where(pick < dense, 0.95, torch.where(pick < numbers, torch.full_like(few, 0.01), few))
    out = torch.empty((rows, -(-vocab // 32)), dtype=torch.int32, device=dev)
    for lo in range(0, rows, 256):
        bits = torch.rand((min(256, rows - lo), vocab), generator=gen, device=dev) < share[lo:lo + 256, None]
        bits[:, vocab - 1] |= pick[lo:lo + 256] > 0.97          # the end of the text: some rows allow little else
        out[lo:lo + 256] = _pack(bits)
    return out


def _logits(case, gen, dev):
    """Rows as a language model's head gives them: a broad mass and some dozens of tokens that stand out."""
    rows, vocab = case["rows"], case["vocab"]
    x = torch.empty((rows, case["stride"]), dtype=_TYPES[case["dtype"]], device=dev)[:, :vocab]
    for lo in range(0, rows, 512):
        part = torch.randn((min(512, rows - lo), vocab), generator=gen, device=dev) * 2
        at = torch.randint(vocab, (part.shape[0], 48), generator=gen, device=dev)
        part.scatter_reduce_(1, at, 4 + 10 * torch.rand(at.shape, generator=gen, device=dev), "amax")
        x[lo:lo + 512] = part.to(x.dtype)
    return x


@functools.lru_cache(maxsize=None)
def _library(vocab, rows):
    """The handle that a server keeps: a grammar with this vocabulary, and the buffers of so many sequences."""
    import numpy as np
    from paper_2506_03887_amd import Pre3
    text = np.append(np.resize(np.frombuffer(b"abcde", dtype=np.uint8), vocab - 1), np.uint8(0))
    lib = Pre3("S ::= S X | X\nX ::= [a-e]\n", text, np.append(np.arange(vocab), vocab - 1), vocab - 1, stack_cap=8)
    i32 = functools.partial(torch.zeros, dtype=torch.int32, device="cuda")
    lib.bind_state(i32(rows), i32((rows, 8)), i32(rows) + 1, i32(rows))
    return lib


def prepare(case, seed):
    dev = torch.device("cuda")
    rows, vocab = case["rows"], case["vocab"]
    gen = torch.Generator(device=dev).manual_seed(seed)
    logits = _logits(case, gen, dev)
    mask = _mask(case["mask"], rows, vocab, gen, dev)
    state = dict(case=case, logits=logits, mask=mask)

    def uniform(lo=0.0, hi=1.0):
        return lo + (hi - lo) * torch.rand(rows, generator=gen, device=dev)

    if case["op"] == "sample":
        f = case["filters"]
        mixed = f == "mixed"
        temperature = uniform(0.6, 1.2)
        if mixed:                                               # every eighth request decodes greedily
            temperature = torch.where(uniform() < 0.125, torch.zeros_like(temperature), temperature)
        top_k = (5 + 200 * uniform() ** 2).to(torch.int32)
        state.update(
            uniform=torch.rand(rows, generator=gen, device=dev), temperature=temperature,
            top_k=torch.where(uniform() < 0.4, torch.zeros_like(top_k), top_k) if mixed else top_k if f == "top_k" else None,
            top_p=torch.where(uniform() < 0.4, torch.ones_like(temperature), uniform(0.8, 0.98)) if mixed else uniform(0.85, 0.98) if f == "top_p" else None,
            min_p=torch.where(uniform() < 0.5, torch.zeros_like(temperature), uniform(0.01, 0.1)) if mixed else uniform(0.01, 0.1) if f == "min_p" else None)
        if own:
            state.update(lib=_library(vocab, rows), tokens=torch.empty(rows, dtype=torch.int32, device=dev),
                         logprobs=torch.empty(rows, device=dev), kept=torch.empty(rows, dtype=torch.int32, device=dev))
        return state
    # the teacher is the student with noise; a tenth of the rows (a question's tokens) teach nothing; weights of the rows as a mean has them
    ids = torch.empty((rows, case["k"]), dtype=torch.int32, device=dev)
    values = torch.empty((rows, case["k"]), dtype=torch.bfloat16, device=dev)
    for lo in range(0, rows, 256):
        part = logits[lo:lo + 256].float()
        part += 2 * torch.randn(part.shape, generator=gen, device=dev)
        if mask is not None:
            part.masked_fill_(~_unpack(mask[lo:lo + 256], vocab), -math.inf)
        best, at = part.topk(case["k"], dim=1)
        best = best.to(values.dtype)
        ids[lo:lo + 256] = torch.where(best > -math.inf, at, torch.full_like(at, -1))
        values[lo:lo + 256] = best
    nothing = uniform() < 0.1
    ids[nothing] = -1
    state.update(ids=ids, values=values, weight=uniform(0.5, 1.5) / rows * 100)
    if case["form"] == "step":
        logits.requires_grad_()
    return state


# ------------------------------------------------------------------------------------------------- one pass

def run(state):
    if state["case"]["op"] == "sample":
        return _run_sample(state) if own else _plain_sample(state)
    return _run_distill(state) if own else _plain_distill(state)


def _run_sample(s):
    s["lib"].apply_mask_sample(s["logits"], s["mask"], s["uniform"], s["tokens"], out_logprobs=s["logprobs"], out_kept=s["kept"],
                               temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return dict(tokens=s["tokens"], logprobs=s["logprobs"], kept=s["kept"])


def _run_distill(s):
    from paper_2506_03887_amd import distill_loss, distill_loss_grad
    tau = s["case"]["tau"]
    if s["case"]["form"] == "step":
        loss = distill_loss(s["logits"], s["ids"], s["values"], s["mask"], temperature=tau)
        grad, = torch.autograd.grad(loss, s["logits"], s["weight"])
        return dict(loss=loss.detach(), grad=grad)
    loss, grad = distill_loss_grad(s["logits"], s["ids"], s["values"], s["mask"], temperature=tau, row_weight=s["weight"])
    return dict(loss=loss, grad=grad)


def _plain_sample(s):
    x, vocab = s["logits"].float(), s["case"]["vocab"]
    candidate = ~torch.isnan(x)
    if s["mask"] is not None:
        candidate &= _unpack(s["mask"], vocab)
    x = torch.where(candidate, x, torch.full_like(x, -math.inf)) + 0.0      # (-0 and +0 are equal)
    best_first, ids = torch.sort(x, dim=1, descending=True, stable=True)
    del x
    best = best_first[:, :1].double()
    t = s["temperature"].double()[:, None]
    # weights in 64 bits: a border that the draw falls next to is one of up to the whole vocabulary
    w = torch.exp((best_first.double() - best) / torch.where(t > 0, t, torch.ones_like(t)))
    w = torch.where(best_first == best_first[:, :1], torch.ones_like(w), w)
    place = torch.arange(vocab, device=w.device)
    n = (best_first > -math.inf).sum(dim=1, keepdim=True)
    if s["top_k"] is not None:
        top_k = s["top_k"].long()[:, None]
        n = torch.where(top_k > 0, torch.minimum(n, top_k), n)
    n = torch.where(t > 0, n, torch.clamp(n, max=1))
    w = torch.where(place < n, w, torch.zeros_like(w))
    upto = torch.cumsum(w, dim=1)
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        inside = (torch.roll(upto, 1, dims=1) < p * upto[:, -1:]) & (place > 0)
        n = torch.where(p < 1, torch.minimum(n, 1 + inside.sum(dim=1, keepdim=True)), n)
    if s["min_p"] is not None:
        likely = (w >= s["min_p"].double()[:, None]).sum(dim=1, keepdim=True)
        n = torch.where(s["min_p"][:, None] > 0, torch.minimum(n, torch.clamp(likely, min=1)), n)
    last = torch.clamp(n - 1, min=0)
    total = upto.gather(1, last)
    at = ((upto <= s["uniform"].double()[:, None] * total) & (place < n)).sum(dim=1, keepdim=True)
    at = torch.minimum(at, last)
    logprob = torch.log(w.gather(1, at) / total)
    # a row whose candidates are all -inf gives the first of them, a row without candidates none
    some, first = candidate.any(dim=1, keepdim=True), candidate.int().argmax(dim=1, keepdim=True)
    dead = n == 0
    token = torch.where(dead, torch.where(some, first, torch.full_like(first, -1)), ids.gather(1, at))
    logprob = torch.where(dead, torch.where(some, torch.zeros_like(logprob), torch.full_like(logprob, -math.inf)), logprob)
    n = torch.where(dead, some.long(), n)
    return dict(tokens=token[:, 0].int(), logprobs=logprob[:, 0].float(), kept=n[:, 0].int())


def _plain_distill(s):
    tau, vocab = s["case"]["tau"], s["case"]["vocab"]
    z = s["logits"].detach().float()
    if s["mask"] is not None:
        z = torch.where(_unpack(s["mask"], vocab), z, torch.full_like(z, -math.inf))
    top = z.amax(dim=1, keepdim=True)
    z = (z - torch.where(top > -math.inf, top, torch.zeros_like(top))) / tau
    e = torch.exp(z)
    total = e.sum(dim=1, keepdim=True, dtype=torch.float64)      # (a long sum, and the loss is a small difference of large numbers)
    at = s["ids"].clamp(min=0).long()
    z_at = z.gather(1, at).double()
    listed_ = (s["ids"] >= 0) & (z_at > -math.inf)               # what the student's row leaves out the teacher does not ask for
    del z
    live = listed_.any(dim=1, keepdim=True)
    t = torch.where(listed_, s["values"].double(), torch.full_like(z_at, -math.inf))
    t = (t - t.amax(dim=1, keepdim=True)) / tau
    q = torch.where(listed_, torch.exp(t), torch.zeros_like(t))
    of = q.sum(dim=1, keepdim=True)
    gap = (t - torch.log(of)) - (z_at - torch.log(total))
    q = q / torch.where(live, of, torch.ones_like(of))
    loss = tau * tau * torch.where(q > 0, q * gap, torch.zeros_like(q)).sum(dim=1)
    grad = e / torch.where(total > 0, total, torch.ones_like(total)).float()
    del e
    grad.scatter_add_(1, at, -q.float())
    grad *= torch.where(live, tau * s["weight"][:, None], torch.zeros_like(top))
    return dict(loss=loss.float(), grad=grad.to(s["logits"].dtype))


# ------------------------------------------------------------------------------------------------- in 64 bits, from the definition

def exact(case, seed):
    s = prepare(case, seed)
    return _exact_sample(s) if case["op"] == "sample" else _exact_distill(s)


def _exact_sample(s):
    """Probabilities, cut and renormalised filter after filter, and the point of their distribution function that the number hits."""
    vocab = s["case"]["vocab"]
    z = s["logits"].double()
    if s["mask"] is not None:
        z.masked_fill_(~_unpack(s["mask"], vocab), -math.inf)
    order = torch.argsort(-(z + 0.0), dim=1, stable=True)
    z = z.gather(1, order)
    t = s["temperature"].double()[:, None]
    greedy = t <= 0
    p = torch.softmax(z / torch.where(greedy, torch.ones_like(t), t), dim=1)
    rank = torch.arange(1, vocab + 1, device=p.device)

    def cut(p, keep):
        p = p * keep
        return p / p.sum(dim=1, keepdim=True)

    p = cut(p, (rank == 1) | ~greedy)
    if s["top_k"] is not None:
        k = s["top_k"][:, None]
        p = cut(p, (rank <= k) | (k <= 0))
    keep = p > 0
    if s["top_p"] is not None:
        limit = s["top_p"].double()[:, None]
        ahead = torch.cat([torch.zeros_like(limit), torch.cumsum(p, dim=1)[:, :-1]], dim=1)
        keep &= (ahead < limit) | (limit >= 1) | (rank == 1)
    if s["min_p"] is not None:
        keep &= p >= s["min_p"].double()[:, None] * p[:, :1]
    alive = torch.isfinite(z[:, :1])
    kept = torch.where(alive, keep.sum(dim=1, keepdim=True), torch.zeros_like(alive, dtype=torch.long))
    p = torch.where(keep, p, torch.zeros_like(p))
    p = torch.where(alive, p / p.sum(dim=1, keepdim=True), torch.zeros_like(p))
    cdf = torch.cumsum(p, dim=1).contiguous()
    at = torch.searchsorted(cdf, s["uniform"].double()[:, None].contiguous(), right=True)
    at = torch.minimum(at, torch.clamp(kept - 1, min=0))
    token = torch.where(alive, order.gather(1, at), torch.full_like(at, -1))
    return dict(tokens=token[:, 0].int(), logprobs=torch.log(p.gather(1, at))[:, 0], kept=kept[:, 0].int())


def _exact_distill(s):
    """The loss as a divergence of two distributions over the vocabulary, and its derivative."""
    tau, vocab, rows = s["case"]["tau"], s["case"]["vocab"], s["case"]["rows"]
    logits = s["logits"].detach()
    losses, grads = [], []
    for lo in range(0, rows, 1024):
        x = logits[lo:lo + 1024].double()
        allowed = torch.ones_like(x, dtype=torch.bool) if s["mask"] is None else _unpack(s["mask"][lo:lo + 1024], vocab)
        x = x.masked_fill(~allowed, -math.inf)
        logp = torch.log_softmax(x / tau, dim=1)
        ids, values = s["ids"][lo:lo + 1024].long(), s["values"][lo:lo + 1024].double()
        ok = (ids >= 0) & allowed.gather(1, ids.clamp(min=0))
        none = ~ok.any(dim=1, keepdim=True)
        logq = torch.log_softmax(values.masked_fill(~ok & ~none, -math.inf) / tau, dim=1)
        q = torch.exp(logq).masked_fill(~ok, 0)
        gap = (logq - logp.gather(1, ids.clamp(min=0))).masked_fill(~ok, 0)
        losses.append(tau ** 2 * (q * gap).sum(dim=1))
        target = torch.zeros_like(x).scatter_add_(1, ids.clamp(min=0), q)
        slope = torch.exp(logp).sub_(target).mul_(tau * s["weight"][lo:lo + 1024, None].double())
        grads.append(slope.masked_fill_(none | ~allowed, 0))
    return dict(loss=torch.cat(losses), grad=torch.cat(grads))


def work(case):
    """The logits read once, for the loss the gradient written once, the mask's bits; the lists and the rows' numbers are small beside
    that.  An exponential and a few operations a token."""
    pairs = case["rows"] * case["vocab"]
    size = _TYPES[case["dtype"]].itemsize * (1 if case["op"] == "sample" else 2)
    mask = 0 if case["mask"] == "none" else pairs / 8
    lists = 24 * case["rows"] if case["op"] == "sample" else case["rows"] * (6 * case["k"] + 8)
    return {"bytes": pairs * size + mask + lists, "flops": pairs * (4 if case["op"] == "sample" else 8)}
