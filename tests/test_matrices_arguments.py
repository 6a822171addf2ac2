"""What the calls on a model's table and head refuse, in Python and at the C ABI, before anything reaches the GPU (no GPU needed)."""
import ctypes as c

import pytest
import torch

import paper_2506_03887_amd as P
from paper_2506_03887_amd import binding

f32, i32 = torch.float32, torch.int32


def zeros(*shape, dtype=f32):
    return torch.zeros(shape, dtype=dtype)


EMBED = dict(weight=zeros(9, 6), tokens=zeros(4, dtype=i32))
HEAD = dict(hidden=zeros(4, 6), weight=zeros(40, 6), targets=zeros(4, dtype=i32), bitmask=None)
LOGITS = dict(hidden=zeros(4, 6), weight=zeros(40, 16, dtype=torch.int8)[:, :6], scale=zeros(40), bitmask=None)

# call, its arguments, what is wrong with one of them; a tensor that fits but lies in host memory is the last thing that is looked at
REFUSED = [
    ("embed", EMBED, dict(weight=zeros(9)), AssertionError), ("embed", EMBED, dict(weight=zeros(6, 9).t()), AssertionError), ("embed", EMBED, dict(weight=zeros(0, 6)), AssertionError),
    ("embed", EMBED, dict(weight=zeros(1, 6).expand(9, 6)), AssertionError), ("embed", EMBED, dict(tokens=zeros(4, 4, dtype=i32)[:, 1]), AssertionError),
    ("embed", EMBED, dict(weight=zeros(9, 6, dtype=torch.float64)), TypeError), ("embed", EMBED, dict(), TypeError),
    ("head_loss", HEAD, dict(hidden=zeros(4, 5)), AssertionError), ("head_loss", HEAD, dict(hidden=zeros(6, 4).t()), AssertionError), ("head_loss", HEAD, dict(targets=zeros(3, dtype=i32)), AssertionError),
    ("head_loss", HEAD, dict(hidden=zeros(1, 6).expand(4, 6)), AssertionError), ("head_loss", HEAD, dict(weight=zeros(1, 6).expand(40, 6)), AssertionError),
    ("head_loss", HEAD, dict(weight=zeros(0, 6)), AssertionError), ("head_loss", HEAD, dict(), TypeError),
    ("head_loss_grad", HEAD, dict(targets=zeros(8, dtype=i32)[::2]), AssertionError), ("head_loss_grad", HEAD, dict(), TypeError),
    ("quantise_rows", dict(x=zeros(4, 6)), dict(x=zeros(6, 4).t()), AssertionError), ("quantise_rows", dict(x=zeros(4, 6)), dict(), TypeError),
    ("head_logits", LOGITS, dict(weight=zeros(40, 6, dtype=torch.int8)), AssertionError), ("head_logits", LOGITS, dict(scale=zeros(39)), AssertionError),
    ("head_logits", LOGITS, dict(hidden=zeros(4, 7)), AssertionError), ("head_logits", LOGITS, dict(weight=zeros(40, 24, dtype=torch.int8)[:, :6]), AssertionError), ("head_logits", LOGITS, dict(), TypeError),
]


@pytest.mark.parametrize("at", range(len(REFUSED)))
def test_tensors_that_do_not_fit(at):
    call, good, bad, error = REFUSED[at]
    with pytest.raises(error):
        getattr(P, call)(**{**good, **bad})


@pytest.mark.parametrize("call", ["embed", "head_loss", "head_loss_grad", "quantise_rows", "head_logits"])
def test_a_forked_process_is_refused(call, monkeypatch):
    binding.load()
    P.head_loss
    monkeypatch.setattr(binding, "_in_bad_fork", lambda: True, raising=False)
    monkeypatch.setattr(torch.cuda, "_is_in_bad_fork", lambda: True)
    good = {"embed": EMBED, "head_loss": HEAD, "head_loss_grad": HEAD, "quantise_rows": dict(x=zeros(4, 6)), "head_logits": LOGITS}[call]
    with pytest.raises(RuntimeError, match="forked"):
        getattr(P, call)(**good)


class Embedding(c.Structure):
    _fields_ = [("table", c.c_void_p), ("ids", c.c_void_p), ("table_stride", c.c_int64), ("type", c.c_int32), ("id_bytes", c.c_int32), ("rows", c.c_int32), ("vocab", c.c_int32),
                ("dim", c.c_int32), ("scale", c.c_float)]


class Head(c.Structure):
    _fields_ = [(n, c.c_void_p) for n in ("hidden", "weight", "targets", "bitmask")] + [("hidden_stride", c.c_int64), ("weight_stride", c.c_int64)] + \
               [(n, c.c_int32) for n in ("type", "target_bytes", "rows", "vocab", "dim")] + [("workspace", c.c_void_p), ("workspace_bytes", c.c_int64), ("kept", c.c_void_p)]


class Head8(c.Structure):
    _fields_ = [(n, c.c_void_p) for n in ("hidden", "weight", "weight_scale", "bitmask")] + [("hidden_stride", c.c_int64), ("weight_stride", c.c_int64)] + \
               [(n, c.c_int32) for n in ("type", "rows", "vocab", "dim")] + [("workspace", c.c_void_p), ("workspace_bytes", c.c_int64)]


NOWHERE = 1 << 20                                       # an address that is never followed
BADARG, LIMIT = binding.E_BADARG, binding.E_LIMIT


def lib():
    lib = binding.load()
    p, i64, n32 = c.c_void_p, c.c_int64, c.c_int32
    lib.pre3_embed.argtypes = [p, p, i64, p]
    lib.pre3_embed_workspace_bytes.argtypes = [n32, n32]
    lib.pre3_embed_grad.argtypes = [p, p, i64, p, p, i64, p]
    lib.pre3_head_workspace_bytes.argtypes = [p, n32]
    lib.pre3_head_kept_bytes.argtypes = [p]
    lib.pre3_head_loss.argtypes = [p, p, p, p]
    lib.pre3_head_grad.argtypes = [p, p, p, i64, p, i64, p, i64, p]
    lib.pre3_head_loss_grad.argtypes = [p, p, i64, p, p, i64, p, i64, p]
    lib.pre3_quantise_rows.argtypes = [p, n32, i64, n32, n32, p, i64, p, p]
    lib.pre3_head8_workspace_bytes.argtypes = [n32, n32]
    lib.pre3_head8_logits.argtypes = [p, p, i64, p]
    return lib


@pytest.mark.parametrize("wrong,status", [(dict(table=None), BADARG), (dict(table=NOWHERE + 1), BADARG), (dict(ids=None), BADARG), (dict(ids=NOWHERE + 2), BADARG), (dict(table_stride=7), BADARG),
                                          (dict(type=3), BADARG), (dict(id_bytes=2), BADARG), (dict(rows=-1), BADARG), (dict(vocab=0), BADARG), (dict(dim=0), BADARG),
                                          (dict(rows=(1 << 22) + 1), LIMIT), (dict(vocab=(1 << 22) + 1), LIMIT), (dict(dim=65537, table_stride=65537), LIMIT)])
def test_embedding_at_the_c_abi(wrong, status):
    e = Embedding(**{**dict(table=NOWHERE, ids=NOWHERE, table_stride=8, type=0, id_bytes=4, rows=3, vocab=9, dim=8, scale=1.0), **wrong})
    assert lib().pre3_embed(c.byref(e), NOWHERE, max(8, e.dim), None) == status
    if "table" not in wrong and "table_stride" not in wrong:
        assert lib().pre3_embed_grad(c.byref(e), NOWHERE, max(8, e.dim), NOWHERE, NOWHERE, 1 << 40, None) == status


@pytest.mark.parametrize("type,vocab,dim,status", [(0, 1 << 18, 65536, BADARG), (0, (1 << 18) + 1, 65536, LIMIT), (2, (1 << 22), 2049, LIMIT), (2, 1 << 22, 2048, BADARG)])
def test_gradients_of_tables_beyond_a_launch(type, vocab, dim, status):
    # (the largest that are taken get as far as the null pointer)
    e = Embedding(NOWHERE, NOWHERE, dim, type, 4, 3, vocab, dim, 1.0)
    assert lib().pre3_embed_grad(c.byref(e), NOWHERE, dim, None, NOWHERE, 1 << 40, None) == status


@pytest.mark.parametrize("rows,dim,status", [(1 << 20, 1 << 14, BADARG), (1 << 20, (1 << 14) + 1, LIMIT), (1 << 18, 1 << 16, BADARG), ((1 << 18) + 1, 1 << 16, LIMIT)])
def test_hidden_states_beyond_a_launch(rows, dim, status):
    h = Head(NOWHERE, NOWHERE, NOWHERE, None, dim, dim, 0, 4, rows, 9, dim, NOWHERE, 1 << 50)
    assert lib().pre3_head_loss(c.byref(h), None, None, None) == status
    assert lib().pre3_head_loss_grad(c.byref(h), None, 0, None, NOWHERE, dim, NOWHERE, dim, None) == status


def test_embedding_outputs_and_workspaces_at_the_c_abi():
    e = Embedding(NOWHERE, NOWHERE, 8, 0, 4, 3, 9, 8, 1.0)
    need = lib().pre3_embed_workspace_bytes(3, 8)
    assert need > 0 and lib().pre3_embed_workspace_bytes(-1, 8) == BADARG and lib().pre3_embed_workspace_bytes(3, 0) == BADARG
    assert lib().pre3_embed(None, NOWHERE, 8, None) == BADARG and lib().pre3_embed(c.byref(e), None, 8, None) == BADARG and lib().pre3_embed(c.byref(e), NOWHERE, 7, None) == BADARG
    for args in ((None, 8, NOWHERE, NOWHERE, need), (NOWHERE, 7, NOWHERE, NOWHERE, need), (NOWHERE, 8, None, NOWHERE, need), (NOWHERE, 8, NOWHERE, None, need),
                 (NOWHERE, 8, NOWHERE, NOWHERE, need - 1), (NOWHERE, 8, NOWHERE, NOWHERE + 8, need)):
        assert lib().pre3_embed_grad(c.byref(e), *args, None) == BADARG, args
    e.rows = 0
    assert lib().pre3_embed(c.byref(e), None, 8, None) == 0


@pytest.mark.parametrize("wrong,status", [(dict(hidden=None), BADARG), (dict(weight=NOWHERE + 1), BADARG), (dict(targets=NOWHERE + 2), BADARG), (dict(bitmask=NOWHERE + 2), BADARG), (dict(kept=NOWHERE + 8), BADARG),
                                          (dict(hidden_stride=7), BADARG), (dict(weight_stride=7), BADARG), (dict(type=-1), BADARG), (dict(target_bytes=1), BADARG), (dict(rows=-1), BADARG),
                                          (dict(vocab=0), BADARG), (dict(dim=0), BADARG), (dict(rows=(1 << 20) + 1), LIMIT), (dict(vocab=(1 << 21) + 1), LIMIT), (dict(dim=65537), LIMIT)])
def test_heads_at_the_c_abi(wrong, status):
    h = Head(**{**dict(hidden=NOWHERE, weight=NOWHERE, targets=NOWHERE, hidden_stride=8, weight_stride=8, type=0, target_bytes=4, rows=3, vocab=9, dim=8, workspace=NOWHERE,
                       workspace_bytes=1 << 40), **wrong})
    assert lib().pre3_head_workspace_bytes(c.byref(h), 1) == status and lib().pre3_head_kept_bytes(c.byref(h)) == status
    assert lib().pre3_head_loss(c.byref(h), NOWHERE, None, None) == status
    assert lib().pre3_head_grad(c.byref(h), NOWHERE, None, 0, NOWHERE, 8, NOWHERE, 8, None) == status
    assert lib().pre3_head_loss_grad(c.byref(h), None, 0, NOWHERE, NOWHERE, 8, NOWHERE, 8, None) == status


def test_head_outputs_and_workspaces_at_the_c_abi():
    h = Head(NOWHERE, NOWHERE, NOWHERE, None, 8, 8, 0, 4, 3, 9, 8, NOWHERE, 0)
    loss_needs, needs = (lib().pre3_head_workspace_bytes(c.byref(h), g) for g in (0, 1))
    assert 0 < loss_needs <= needs
    assert lib().pre3_head_kept_bytes(c.byref(h)) == 3 * 16 * 4                              # of few rows the logits, whole pieces of 16
    many = Head(NOWHERE, NOWHERE, NOWHERE, None, 4096, 4096, 0, 4, 4096, 128256, 4096, NOWHERE, 0)
    assert lib().pre3_head_kept_bytes(c.byref(many)) == 0
    h.workspace_bytes = loss_needs - 1
    assert lib().pre3_head_loss(c.byref(h), NOWHERE, None, None) == BADARG
    h.workspace_bytes = needs - 1
    assert lib().pre3_head_grad(c.byref(h), NOWHERE, None, 0, NOWHERE, 8, None, 8, None) == BADARG
    h.workspace_bytes, h.workspace = needs, NOWHERE + 128
    assert lib().pre3_head_loss(c.byref(h), NOWHERE, None, None) == BADARG
    h.workspace = NOWHERE
    assert lib().pre3_head_loss(c.byref(h), None, None, None) == BADARG and lib().pre3_head_loss(c.byref(h), NOWHERE, NOWHERE + 4, None) == BADARG
    grad = lib().pre3_head_grad
    for args in ((None, None, 0, NOWHERE, 8, NOWHERE, 8), (NOWHERE, None, -1, NOWHERE, 8, NOWHERE, 8), (NOWHERE, None, 0, NOWHERE, 7, NOWHERE, 8), (NOWHERE, None, 0, NOWHERE, 8, NOWHERE, 7),
                 (NOWHERE, None, 0, NOWHERE + 1, 8, NOWHERE, 8), (NOWHERE, NOWHERE + 2, 1, NOWHERE, 8, NOWHERE, 8)):
        assert grad(c.byref(h), *args, None) == BADARG, args
    assert grad(c.byref(h), NOWHERE, None, 0, None, 8, None, 8, None) == 0                   # nothing wanted
    h.rows = 0
    assert lib().pre3_head_loss(c.byref(h), None, None, None) == 0 and grad(c.byref(h), None, None, 0, NOWHERE, 8, None, 8, None) == 0


@pytest.mark.parametrize("wrong,status", [(dict(hidden=None), BADARG), (dict(weight=NOWHERE + 8), BADARG), (dict(weight_scale=None), BADARG), (dict(bitmask=NOWHERE + 1), BADARG),
                                          (dict(hidden_stride=7), BADARG), (dict(weight_stride=24), BADARG), (dict(weight_stride=1 << 23), BADARG), (dict(type=7), BADARG), (dict(rows=-1), BADARG),
                                          (dict(vocab=0), BADARG), (dict(dim=0), BADARG), (dict(rows=(1 << 20) + 1), LIMIT), (dict(workspace=None), BADARG), (dict(workspace_bytes=15), BADARG)])
def test_heads_in_8_bits_at_the_c_abi(wrong, status):
    h = Head8(**{**dict(hidden=NOWHERE, weight=NOWHERE, weight_scale=NOWHERE, hidden_stride=8, weight_stride=16, type=0, rows=3, vocab=9, dim=8, workspace=NOWHERE, workspace_bytes=1 << 40), **wrong})
    assert lib().pre3_head8_logits(c.byref(h), NOWHERE, 9, None) == status


def test_rows_in_8_bits_at_the_c_abi():
    call = lib().pre3_quantise_rows
    good = dict(x=NOWHERE, type=0, x_stride=8, rows=3, dim=8, out=NOWHERE, out_stride=16, scale=NOWHERE)
    for wrong in (dict(x=None), dict(x=NOWHERE + 1), dict(type=9), dict(x_stride=7), dict(rows=-1), dict(dim=0), dict(out=None), dict(out=NOWHERE + 8), dict(out_stride=8), dict(scale=None)):
        assert call(*{**good, **wrong}.values(), None) == BADARG, wrong
    assert call(*{**good, **dict(dim=65537, x_stride=65537, out_stride=65552)}.values(), None) == LIMIT
    assert call(*{**good, **dict(rows=(1 << 22) + 1)}.values(), None) == LIMIT
    assert call(*{**good, **dict(rows=0)}.values(), None) == 0
    h = Head8(hidden=NOWHERE, weight=NOWHERE, weight_scale=NOWHERE, hidden_stride=8, weight_stride=16, rows=3, vocab=9, dim=8, workspace=NOWHERE, workspace_bytes=1 << 40)
    assert lib().pre3_head8_logits(c.byref(h), None, 9, None) == BADARG and lib().pre3_head8_logits(c.byref(h), NOWHERE, 8, None) == BADARG
    assert lib().pre3_head8_workspace_bytes(3, 8) > 0 and lib().pre3_head8_workspace_bytes(-1, 8) == BADARG


def test_tangents_are_refused():
    import torch.autograd.forward_ad as fwd
    with fwd.dual_level():
        x = fwd.make_dual(zeros(4, 6), torch.ones(4, 6))
        # (tensors in host memory are refused first: what is checked is that no call takes a tangent and loses it)
        for call in (lambda: P.head_loss(x, zeros(40, 6), zeros(4, dtype=i32)), lambda: P.head_logits(x, LOGITS["weight"], zeros(40)), lambda: P.embed(x, zeros(2, dtype=i32))):
            with pytest.raises((TypeError, NotImplementedError)):
                call()
