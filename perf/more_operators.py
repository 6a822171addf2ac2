"""What is measured of the operators on a model's two vocabulary-sized matrices: the table that tokens are looked up in, and the head whose
product with the hidden states gives the logits that mask, sampler and loss work on.

  embed     rows of the table by token, times a scale ("lookup"); with the table's gradient, through autograd ("step")
  loss      the cross entropy of a target token a row in the logits hidden @ weight.T behind the mask: the losses alone ("score"), with the
            gradients of hidden states and weights through autograd ("step"), or all three in one call ("pass")
  logits    the logits of hidden states against weights of 8 bits with a scale a token, the hidden states quantised row by row on the
            way, -inf where the mask has no bit

A case names
  op, form  as above
  dtype     of the table, the hidden states and weights, the logits: bf16 | f16 | f32
  rows, vocab, dim (elements of a token's row)
  mask      none | text (rows inside a string allow nearly everything, others a number's or a structure's tokens) | schema (a
            handful of tokens in most rows)
  taught    of loss: the rows that have a target; the others (a question's tokens, padding) teach nothing
"""
import math

import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _embed(name, form, dtype, rows, vocab, dim):
    case = dict(op="embed", form=form, dtype=dtype, rows=rows, vocab=vocab, dim=dim)
    return dict(case, name=name) if name else case


def _loss(name, form, dtype, rows, vocab, dim, mask, taught):
    case = dict(op="loss", form=form, dtype=dtype, rows=rows, vocab=vocab, dim=dim, mask=mask, taught=taught)
    return dict(case, name=name) if name else case


def _logits(name, dtype, rows, vocab, dim, mask):
    case = dict(op="logits", dtype=dtype, rows=rows, vocab=vocab, dim=dim, mask=mask)
    return dict(case, name=name) if name else case


def listed():
    return [
        # a decode step of four sequences on the smallest vocabulary: a launch's latency
        _embed("embed lookup 4 small f32", "lookup", "f32", 4, 513, 512),
        # a batch of questions on their way into a model
        _embed("embed lookup 16384", "lookup", "bf16", 16384, 128256, 4096),
        # a training step's lookup in 16-bit floats, rows of odd length
        _embed("embed step 5000 f16", "step", "f16", 5000, 50257, 1001),
        # a training step of eight texts of 4,096 tokens: common tokens thousands of times, most of the table not at all
        _embed("embed step 32768", "step", "bf16", 32768, 128256, 4096),
        # one document's next token, scored
        _loss("loss score 1", "score", "bf16", 1, 128256, 4096, "text", 1),
        # a toy model
        _loss("loss step 64 small f32", "step", "f32", 64, 513, 512, "text", 56),
        # one text of odd length, no grammar, rows off 16-byte boundaries
        _loss("loss step 300 f16", "step", "f16", 300, 100003, 1001, "none", 300),
        # a small model's batch of constrained answers, a third of the tokens the question's
        _loss("loss step 2048", "step", "bf16", 2048, 32000, 2048, "text", 1400),
        # the largest: a training step of eight answers of 512 tokens
        _loss("loss pass 4096", "pass", "bf16", 4096, 128256, 4096, "text", 3700),
        # one user's document: the latency of reading the head
        _logits("logits 1", "bf16", 1, 128256, 4096, "none"),
        # a small server's step under grammars, in 16-bit floats, odd sizes
        _logits("logits 96 f16", "f16", 96, 100003, 1001, "text"),
        # structured output, a large batch and vocabulary
        _logits("logits 512", "bf16", 512, 152064, 4096, "schema"),
    ]


def _spread(rng, lo, hi):
    """An integer of lo..hi, spread over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    vocab, dim = _spread(rng, 100, 200_000), _spread(rng, 64, 8192)
    if rng.random() < 0.6:
        dim = -(-dim // 64) * 64                                # what models have; the rest are odd
    dtype, mask = rng.choice(("bf16", "bf16", "f16", "f32")), rng.choice(("none", "text", "text", "schema"))
    op = rng.choice(("embed", "loss", "loss", "logits"))
    if vocab * dim > 128256 * 4096:
        vocab = 128256 * 4096 // dim
    if op == "embed":
        return _embed(None, rng.choice(("lookup", "step")), dtype, _spread(rng, 1, min(65536, 32768 * 4096 // dim)), vocab, dim)
    if op == "logits":
        return _logits(None, dtype, _spread(rng, 1, min(1024, 512 * 152064 // vocab)), vocab, dim, mask)
    work = 4096 * 128256 * 4096 // (6 if dtype == "f32" else 1)
    rows = _spread(rng, 1, min(8192, work // (vocab * dim)))
    return _loss(None, rng.choice(("score", "step", "pass")), dtype, rows, vocab, dim, mask, rows - int(rows * rng.choice((0, 0.1, 0.4))))


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


def _mask(kind, rows, vocab, targets, gen, dev):
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
        if targets is not None:                                 # an answer's tokens are allowed, but for one in a hundred that a teacher got wrong
            bits |= (torch.arange(vocab, device=dev) == targets[lo:lo + 256, None]) & ((pick[lo:lo + 256] * 1e4 % 1) > 0.01)[:, None]
        out[lo:lo + 256] = _pack(bits)
    return out


def _tokens(n, vocab, gen, dev):
    """Token ids as texts have them: the i-th one about 1 / (i + 1) as often as the first."""
    u = torch.rand(n, generator=gen, device=dev, dtype=torch.float64)
    return (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp(0, vocab - 1).int()


def prepare(case, seed):
    dev = torch.device("cuda")
    rows, vocab, dim, dtype = case["rows"], case["vocab"], case["dim"], _TYPES[case["dtype"]]
    gen = torch.Generator(device=dev).manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    state = dict(case=case)
    if case["op"] == "embed":
        tokens = _tokens(rows, vocab, gen, dev)
        if rows > 4:                                            # finished sequences and padding have no token
            tokens[torch.rand(rows, generator=gen, device=dev) < 0.02] = -1
        state.update(weight=(0.02 * normal(vocab, dim)).to(dtype), tokens=tokens, scale=math.sqrt(dim))
        if case["form"] == "step":
            state["weight"].requires_grad_()
            state["grad"] = (normal(rows, dim) * (100 / rows)).to(dtype)
        return state
    weight = normal(vocab, dim) * (2 / math.sqrt(dim))          # logits of a spread of 2
    if case["op"] == "logits":
        # a head in 8 bits as it is kept: rows at 16-byte boundaries, a scale each
        top = weight.abs().amax(dim=1)
        scale = top / 127
        kept = torch.zeros((vocab, -(-dim // 16) * 16), dtype=torch.int8, device=dev)
        kept[:, :dim] = (weight * (127 / top)[:, None]).round_()
        state.update(hidden=normal(rows, dim).to(dtype), weight=kept[:, :dim], scale=scale, mask=_mask(case["mask"], rows, vocab, None, gen, dev))
        if own:
            state["out"] = torch.empty((rows, vocab), dtype=dtype, device=dev)
        return state
    targets = _tokens(rows, vocab, gen, dev)
    mask = _mask(case["mask"], rows, vocab, targets, gen, dev)
    # a model that has learnt something: hidden states lean towards their target's weights
    hidden = normal(rows, dim) + 2.5 * weight[targets.long()]
    targets[torch.randperm(rows, generator=gen, device=dev)[case["taught"]:]] = -1
    state.update(hidden=hidden.to(dtype), weight=weight.to(dtype), targets=targets, mask=mask)
    if case["form"] != "score":
        state["row_weight"] = (0.5 + torch.rand(rows, generator=gen, device=dev)) * (100 / rows)
    if case["form"] == "step":
        state["hidden"].requires_grad_()
        state["weight"].requires_grad_()
    return state


# ------------------------------------------------------------------------------------------------- one pass

def run(state):
    op = state["case"]["op"]
    if op == "embed":
        return _run_embed(state) if own else _plain_embed(state)
    if op == "loss":
        return _run_loss(state) if own else _plain_loss(state)
    return _run_logits(state) if own else _plain_logits(state)


def _run_embed(s):
    from paper_2506_03887_amd import embed
    rows = embed(s["weight"], s["tokens"], scale=s["scale"])
    if s["case"]["form"] == "lookup":
        return dict(rows=rows)
    grad, = torch.autograd.grad(rows, s["weight"], s["grad"])
    return dict(rows=rows.detach(), grad=grad)


def _run_loss(s):
    from paper_2506_03887_amd import head_loss, head_loss_grad
    form = s["case"]["form"]
    if form == "pass":
        loss, hidden, weight = head_loss_grad(s["hidden"], s["weight"], s["targets"], s["mask"], row_weight=s["row_weight"])
        return dict(loss=loss, hidden=hidden, weight=weight)
    loss = head_loss(s["hidden"], s["weight"], s["targets"], s["mask"])
    if form == "score":
        return dict(loss=loss)
    hidden, weight = torch.autograd.grad(loss, (s["hidden"], s["weight"]), s["row_weight"])
    return dict(loss=loss.detach(), hidden=hidden, weight=weight)


def _run_logits(s):
    from paper_2506_03887_amd import head_logits
    return dict(logits=head_logits(s["hidden"], s["weight"], s["scale"], s["mask"], out=s["out"]))


def _plain_embed(s):
    weight, at = s["weight"].detach(), s["tokens"].long()
    none = (at < 0) | (at >= len(weight))
    at = torch.where(none, torch.zeros_like(at), at)
    rows = weight[at].float() * s["scale"]
    rows[none] = 0
    out = dict(rows=rows.to(weight.dtype))
    if s["case"]["form"] == "step":
        grad = torch.zeros(weight.shape, device=weight.device)
        grad.index_add_(0, at, torch.where(none[:, None], 0.0, s["grad"].float()))
        out["grad"] = (grad * s["scale"]).to(weight.dtype)
    return out


def _plain_loss(s):
    hidden, weight = s["hidden"].detach().float(), s["weight"].detach().float()
    x = hidden @ weight.T
    if s["mask"] is not None:
        x = torch.where(_unpack(s["mask"], x.shape[1]), x, torch.full_like(x, -math.inf))
    at = s["targets"].long()[:, None]
    there = (at >= 0) & (at < x.shape[1])
    at = torch.where(there, at, torch.zeros_like(at))
    x_at = x.gather(1, at)
    there &= x_at > -math.inf                                   # a target that is not allowed teaches nothing
    top = x.amax(dim=1, keepdim=True)
    e = torch.exp(x - torch.where(top > -math.inf, top, torch.zeros_like(top)))
    del x
    total = e.sum(dim=1, keepdim=True)
    loss = torch.where(there, torch.log(total) - (x_at - top), torch.zeros_like(top))[:, 0]
    if s["case"]["form"] == "score":
        return dict(loss=loss)
    slope = torch.where(there, s["row_weight"][:, None], torch.zeros_like(top))
    e *= slope / torch.where(total > 0, total, torch.ones_like(total))
    e.scatter_add_(1, at, -slope)
    dtype = s["hidden"].dtype
    return dict(loss=loss, hidden=(e @ weight).to(dtype), weight=(e.T @ hidden).to(dtype))


def _plain_logits(s):
    x = s["hidden"].float()
    top = x.abs().amax(dim=1, keepdim=True)
    x = (x * torch.where(top > 0, 127 / top, torch.zeros_like(top))).round()
    x = (x @ s["weight"].float().T) * (top / 127) * s["scale"]
    if s["mask"] is not None:
        x = torch.where(_unpack(s["mask"], x.shape[1]), x, torch.full_like(x, -math.inf))
    return dict(logits=x.to(s["hidden"].dtype))


# ------------------------------------------------------------------------------------------------- in 64 bits, from the definition

def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return {"embed": _exact_embed, "loss": _exact_loss, "logits": _exact_logits}[case["op"]](s)


def _exact_embed(s):
    weight, tokens = s["weight"].detach(), s["tokens"]
    some = torch.nonzero((tokens >= 0) & (tokens < len(weight)))[:, 0]
    rows = torch.zeros((len(tokens), weight.shape[1]), dtype=torch.float64, device=weight.device)
    rows[some] = weight.index_select(0, tokens[some].long()).double() * s["scale"]
    if s["case"]["form"] == "lookup":
        return dict(rows=rows)
    # the rows of a token side by side, their sums as differences of one token's end and the one's before
    order = some[torch.argsort(tokens[some], stable=True)]
    at, count = torch.unique_consecutive(tokens[order].long(), return_counts=True)
    grad = torch.zeros(weight.shape, dtype=torch.float64, device=weight.device)
    for lo in range(0, weight.shape[1], 1024):
        upto = torch.cumsum(s["grad"][order, lo:lo + 1024].double(), dim=0)[torch.cumsum(count, dim=0) - 1]
        upto[1:] -= upto[:-1].clone()
        grad[at, lo:lo + 1024] = upto * s["scale"]
    return dict(rows=rows, grad=grad)


def _exact_loss(s):
    """The negative log-probability of the target in the distribution over the allowed tokens, and its derivative."""
    hidden, weight, vocab = s["hidden"].double(), s["weight"].double(), s["case"]["vocab"]
    losses, slopes, d_weight = [], [], torch.zeros_like(weight)
    for lo in range(0, len(hidden), 1024):
        h, target = hidden[lo:lo + 1024], s["targets"][lo:lo + 1024].long()
        x = h @ weight.T
        if s["mask"] is not None:
            x.masked_fill_(~_unpack(s["mask"][lo:lo + 1024], vocab), -math.inf)
        logp = torch.log_softmax(x, dim=1)
        row = torch.arange(len(h), device=h.device)
        taught = (target >= 0) & torch.isfinite(x[row, target.clamp(min=0)])
        losses.append((-logp[row, target.clamp(min=0)]).masked_fill_(~taught, 0))
        if s["case"]["form"] == "score":
            continue
        slope = torch.exp(logp)
        slope[row, target.clamp(min=0)] -= 1
        slope = slope.mul_(s["row_weight"][lo:lo + 1024, None].double())
        slope[~taught] = 0
        slopes.append(slope @ weight)
        d_weight.addmm_(slope.T, h)
    if s["case"]["form"] == "score":
        return dict(loss=torch.cat(losses))
    return dict(loss=torch.cat(losses), hidden=torch.cat(slopes), weight=d_weight)


def _exact_logits(s):
    """A row's whole numbers are its elements times a factor, both of 32 bits, rounded to 32 bits and then to the nearest whole number."""
    x = s["hidden"].double()
    top = x.abs().max(dim=1).values
    factor = (127 / top).float().double()
    whole = torch.round((x * factor[:, None]).float().double())
    y = torch.mm(whole, s["weight"].double().T)
    y *= (top / 127)[:, None]
    y *= s["scale"].double()[None, :]
    if s["mask"] is not None:
        y.masked_fill_(~_unpack(s["mask"], s["case"]["vocab"]), -math.inf)
    return dict(logits=y)


def work(case):
    """Every input read once, every output written once.  Of the table the rows that are looked up (with `embed`, as many as its tokens are
    likely to name); of the loss the rows that have a target, three products where gradients are asked for."""
    rows, vocab, dim, size = case["rows"], case["vocab"], case["dim"], _TYPES[case["dtype"]].itemsize
    if case["op"] == "embed":
        i = torch.arange(vocab, dtype=torch.float64)
        named = float((1 - (1 - torch.log((i + 2) / (i + 1)) / math.log(vocab + 1)) ** rows).sum())
        moved = (named + rows) * dim * size + 4 * rows
        if case["form"] == "lookup":
            return {"bytes": moved, "flops": rows * dim}
        return {"bytes": moved + (rows + vocab) * dim * size, "flops": 2 * rows * dim + vocab * dim}
    mask = 0 if case["mask"] == "none" else vocab / 8
    if case["op"] == "logits":
        return {"bytes": vocab * (dim + 4) + rows * (dim * size + vocab * size + mask), "flops": 2 * rows * vocab * dim}
    taught = case["taught"]
    once = (taught + vocab) * dim * size
    grads = 0 if case["form"] == "score" else 1
    return {"bytes": once * (1 + grads) + taught * mask + 8 * rows, "flops": taught * vocab * (dim * (6 if grads else 2) + 4)}
