"""Lookups and gradients of many tokens and of the largest vocabulary, against the definition in 64 bits, within the bounds that test_gpu_embed derives."""
import pytest
import torch

from test_gpu_embed import TYPES, check_grad, table_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,rows,vocab,dim,ids", [("bf16", 300001, 32000, 9, torch.int32), ("f32", 262144, 3, 8, torch.int64), ("f16", 100, 1 << 22, 5, torch.int64), ("bf16", 9001, 1 << 22, 1, torch.int32)])
def test_many(dtype, rows, vocab, dim, ids):
    from paper_2506_03887_amd import embed
    print(f"[embed] {dtype} {rows} of {vocab} x {dim}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    table = table_of(dtype, vocab, dim, gen).requires_grad_()
    tokens = torch.randint(-1, vocab + 1, (rows,), generator=gen, device="cuda").to(ids)
    tokens[:3] = torch.tensor([vocab - 1, 0, vocab - 1], device="cuda")
    out = embed(table, tokens, 1.0)
    some = (tokens >= 0) & (tokens < vocab)
    assert torch.equal(out[some], table.detach()[tokens[some].long()]) and not out[~some].any()
    upstream = torch.randn((rows, dim), generator=gen, device="cuda").to(TYPES[dtype])
    got, = torch.autograd.grad(out, table, upstream, retain_graph=True)
    check_grad(got, tokens, upstream, 1.0, vocab, dtype)
    again, = torch.autograd.grad(out, table, upstream)
    assert torch.equal(got, again)
