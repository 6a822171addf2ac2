"""Autograd is told of every tensor that a call is handed and writes, so that a node which has saved it (the distillation's mask and lists, an
embedding's tokens) raises in its backward pass instead of taking the new values for the saved ones (no GPU needed: the library's
functions are stood in for)."""
import numpy as np
import pytest
import torch

from paper_2506_03887_amd import Pre3, apply_mask, binding

B, V = 3, 6


class Answers:
    """A library whose functions all succeed."""

    def __getattr__(self, name):
        return lambda *a: 0


@pytest.fixture
def lib(monkeypatch):
    real = Pre3("S ::= S X | X\nX ::= [a-e]\n", np.frombuffer(b"abcde\0", np.uint8), np.arange(7), 5, stack_cap=8, host_only=True)
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(binding, "_stream_ptr", lambda s: None)
    monkeypatch.setattr(binding, "_lib", Answers())
    of_the_handle = real._lib
    real._lib = Answers()
    yield real
    real._lib = of_the_handle


def tensors(lib):
    i32 = lambda *shape: torch.zeros(shape, dtype=torch.int32)  # noqa: E731
    return dict(tokens=i32(B), out=i32(B), states=i32(B), data=i32(B, 8), length=i32(B), err=i32(B), mask=i32(B, lib.words), ids=i32(B, 2),
                values=torch.zeros((B, 2), dtype=torch.bfloat16), logits=torch.zeros((B, V), dtype=torch.bfloat16), uniform=torch.zeros(B),
                logprobs=torch.zeros(B), kept=i32(B), text=torch.zeros((B, 4), dtype=torch.uint8))


CALLS = {
    "fill_mask": (lambda lib, t: lib.fill_mask(t["states"], t["data"], t["length"], t["mask"]), {"mask"}),
    "fill_apply_mask": (lambda lib, t: lib.fill_apply_mask(t["states"], t["data"], t["length"], t["mask"], t["logits"]), {"mask", "logits"}),
    "advance_static": (lambda lib, t: lib.advance_static(t["tokens"], t["states"], t["data"], t["length"], t["err"]), {"states", "data", "length", "err"}),
    "advance_fill_mask": (lambda lib, t: lib.advance_fill_mask(t["tokens"], t["mask"]), {"mask"}),
    "advance_fill_apply_mask": (lambda lib, t: lib.advance_fill_apply_mask(t["tokens"], t["mask"], t["logits"]), {"mask", "logits"}),
    "advance_fill_argmax": (lambda lib, t: lib.advance_fill_argmax(t["tokens"], t["mask"], t["logits"], t["out"]), {"mask", "out"}),
    "apply_mask_argmax": (lambda lib, t: lib.apply_mask_argmax(t["logits"], t["mask"], t["out"]), {"out"}),
    "apply_mask_topk": (lambda lib, t: lib.apply_mask_topk(t["logits"], t["mask"], t["ids"], t["values"]), {"ids", "values"}),
    "apply_mask_topk, ids": (lambda lib, t: lib.apply_mask_topk(t["logits"], t["mask"], t["ids"]), {"ids"}),
    "apply_mask_sample": (lambda lib, t: lib.apply_mask_sample(t["logits"], t["mask"], t["uniform"], t["out"], t["logprobs"], t["kept"]), {"out", "logprobs", "kept"}),
    "apply_mask_sample, tokens": (lambda lib, t: lib.apply_mask_sample(t["logits"], None, t["uniform"], t["out"]), {"out"}),
    "jump_forward": (lambda lib, t: lib.jump_forward(t["text"], t["length"]), {"text", "length"}),
    "apply_mask": (lambda lib, t: apply_mask(t["logits"], t["mask"], V), {"logits"}),
}


@pytest.mark.parametrize("name", CALLS)
def test_what_a_call_writes_has_a_new_version(lib, name):
    call, written = CALLS[name]
    t = tensors(lib)
    call(lib, t)
    assert {n for n, x in t.items() if x._version} == written


def test_a_tensor_of_inference_mode_has_no_version(lib):
    with torch.inference_mode():
        t = tensors(lib)
    for call, _ in CALLS.values():
        call(lib, t)


def test_a_saved_mask_that_a_call_has_written_is_an_error(lib):
    t = tensors(lib)

    class Keeps(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, mask):
            ctx.save_for_backward(mask)
            return x.sum()

        @staticmethod
        def backward(ctx, g):
            return ctx.saved_tensors[0][:, :1] * g, None

    loss = Keeps.apply(torch.zeros((B, 1), requires_grad=True), t["mask"])
    lib.advance_fill_mask(t["tokens"], t["mask"])
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
