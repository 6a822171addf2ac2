"""What the sampler and the distillation refuse, and how (no GPU)."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2506_03887_amd import Pre3, Pre3Error, binding, distill_loss, distill_loss_grad


@pytest.fixture(scope="module")
def lib():
    return Pre3("S ::= S X | X\nX ::= [a-e]\n", np.frombuffer(b"abcde\0", np.uint8), np.arange(7), 5, stack_cap=8, host_only=True)


def test_sampler_arguments(lib):
    rows = 3
    good = dict(logits=torch.zeros((rows, 8)), bitmask=torch.zeros((rows, lib.words), dtype=torch.int32), uniform=torch.zeros(rows),
                out_tokens=torch.zeros(rows, dtype=torch.int32))
    for change in (dict(logits=torch.zeros((8, rows)).t()), dict(logits=torch.zeros((rows, 5))), dict(logits=torch.zeros(8)), dict(logits=torch.zeros((2, 8))),
                   dict(bitmask=good["bitmask"][:2]), dict(bitmask=torch.zeros((rows, lib.words + 1), dtype=torch.int32)), dict(uniform=torch.zeros(4)),
                   dict(uniform=torch.zeros(6)[::2]), dict(temperature=torch.zeros(2)), dict(top_k=torch.zeros(1, dtype=torch.int32)),
                   dict(out_kept=torch.zeros(5, dtype=torch.int32)), dict(out_logprobs=torch.zeros((rows, 2))[:, 0])):
        with pytest.raises(AssertionError):
            lib.apply_mask_sample(**{**good, **change})
    with pytest.raises(TypeError):                           # host tensors
        lib.apply_mask_sample(**good)


def test_sampler_kinds_of_tensors(lib, monkeypatch):
    """Types are looked at before the library is called (the tensors stand in for device ones)."""
    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(binding, "_stream_ptr", lambda s: None)
    rows = 3
    good = dict(logits=torch.zeros((rows, 8)), bitmask=None, uniform=torch.zeros(rows), out_tokens=torch.zeros(rows, dtype=torch.int32))
    for change in (dict(logits=torch.zeros((rows, 8), dtype=torch.float64)), dict(logits=torch.zeros((rows, 8), dtype=torch.int32)),
                   dict(uniform=torch.zeros(rows, dtype=torch.float64)), dict(top_k=torch.zeros(rows, dtype=torch.int64)), dict(top_p=torch.zeros(rows, dtype=torch.bfloat16)),
                   dict(out_tokens=torch.zeros(rows, dtype=torch.int64))):
        with pytest.raises(TypeError):
            lib.apply_mask_sample(**{**good, **change})
    with pytest.raises(Pre3Error):                           # a handle without device tables
        lib.apply_mask_sample(**good)


def c_distill(**change):
    d = dict(logits=4096, bitmask=4096, teacher_ids=4096, teacher_logits=4096, row_stride=10, logits_type=0, teacher_type=0, rows=4, vocab=10, k=3,
             temperature=1.0)
    d.update(change)
    return binding._Distill(**d)


@pytest.mark.parametrize("change", [dict(logits=None), dict(teacher_ids=None), dict(teacher_logits=None), dict(row_stride=9), dict(logits_type=3),
                                    dict(teacher_type=-1), dict(rows=-1), dict(vocab=0), dict(k=0), dict(k=257), dict(temperature=0.0),
                                    dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-30),
                                    dict(logits=4097), dict(logits=4098, logits_type=2), dict(bitmask=4098), dict(teacher_logits=4097)])
def test_distillation_c_arguments(change):
    """No pointer of these is followed: the calls end before a launch."""
    lib, d = binding.load(), c_distill(**change)
    assert lib.pre3_distill_loss(ctypes.byref(d), 1 << 20, 1 << 20, None) == binding.E_BADARG
    assert lib.pre3_distill_grad(ctypes.byref(d), 1 << 20, None, 0, 1 << 20, 10, None) == binding.E_BADARG
    assert lib.pre3_distill_loss_grad(ctypes.byref(d), None, 0, 1 << 20, 1 << 20, 10, None) == binding.E_BADARG


def test_distillation_c_outputs():
    lib, d = binding.load(), c_distill()
    far, ref = 1 << 20, ctypes.byref(d)
    assert lib.pre3_distill_loss(None, far, far, None) == binding.E_BADARG
    assert lib.pre3_distill_loss(ref, None, far, None) == binding.E_BADARG
    assert lib.pre3_distill_loss(ref, far, far + 4, None) == binding.E_BADARG
    assert lib.pre3_distill_grad(ref, None, None, 0, far, 10, None) == binding.E_BADARG
    for grad, stride, weight_stride in ((None, 10, 0), (far, 9, 0), (far + 1, 10, 0), (far, 10, -1), (4096 + 2, 10, 0), (4096 + 60, 10, 0), (4096 - 40, 10, 0),
                                        (4096, 11, 0)):      # overlapping the logits, and in their place with another stride
        assert lib.pre3_distill_grad(ref, far, None, weight_stride, grad, stride, None) == binding.E_BADARG
        assert lib.pre3_distill_loss_grad(ref, None, weight_stride, far, grad, stride, None) == binding.E_BADARG
    empty = c_distill(rows=0, logits=None, teacher_ids=None, teacher_logits=None)
    assert lib.pre3_distill_loss(ctypes.byref(empty), None, None, None) == binding.PRE3_OK
    assert lib.pre3_distill_loss_grad(ctypes.byref(empty), None, 0, None, None, 0, None) == binding.PRE3_OK


def test_distillation_arguments():
    x, ids, values = torch.zeros((3, 40)), torch.zeros((3, 2), dtype=torch.int32), torch.zeros((3, 2))
    mask = torch.zeros((3, 2), dtype=torch.int32)
    for bad in ((x[0], ids, values, None), (x.t(), ids, values, None), (x, ids[:2], values[:2], None), (x, ids, values[:, :1], None), (x, ids[:, 0], values[:, 0], None),
                (x, ids, values, mask[:, :1]), (x, ids, values, mask[:2]), (x, ids.t().contiguous().t(), values, None)):
        for call in (distill_loss, distill_loss_grad):
            with pytest.raises(AssertionError):
                call(*bad)
    for call in (distill_loss, distill_loss_grad):
        with pytest.raises(TypeError):                       # host tensors
            call(x, ids, values, mask)


def test_distillation_workspace():
    """Few long rows go over several blocks, a pair of numbers for each of a row and one for the row."""
    bytes_of = binding.load().pre3_distill_workspace_bytes
    assert bytes_of(160, 24575) == bytes_of(161, 24576) == bytes_of(4096, 128256) == bytes_of(0, 128256) == 0
    assert bytes_of(160, 24576) == 160 * (3 + 1) * 8
    assert bytes_of(1, 128256) == (15 + 1) * 8
    assert bytes_of(1, 2 ** 20) == (64 + 1) * 8
    assert bytes_of(100, 128256) == 100 * (5 + 1) * 8


def test_the_stride_of_a_single_row_may_be_anything(lib, monkeypatch):
    """A column turned into a row is contiguous, with a stride that says nothing."""
    seen = []

    class Library:
        def pre3_apply_mask_sample(self, h, logits, kind, stride, *more):
            seen.append(stride)
            return 0

    monkeypatch.setattr(torch.Tensor, "is_cuda", True, raising=False)
    monkeypatch.setattr(binding, "_stream_ptr", lambda s: None)
    monkeypatch.setattr(lib, "_lib", Library())
    for logits in (torch.zeros((8, 1)).t(), torch.zeros((1, 8)), torch.zeros((1, 3, 8))[:, -1], torch.zeros((2, 8, 1))[0].t()):
        lib.apply_mask_sample(logits, None, torch.zeros(1), torch.zeros(1, dtype=torch.int32))
    assert [s >= 8 for s in seen] == [True] * 4
    lib.apply_mask_sample(torch.zeros((3, 9))[:, :7], None, torch.zeros(3), torch.zeros(3, dtype=torch.int32))
    assert seen[-1] == 9
