"""Lookup by tokens and its gradient against the definition in 64 bits: tables and batches of every proportion, tokens that fill the
batch, that never occur, that lie outside the table, both token types, every element type, odd widths, strides and offsets.

Tolerance of a sum of c tokens: c - 1 additions, the factor and at most eight shares joined: (c + 10) 2^-24 of the sum of
absolute terms, and one rounding to the type."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import embed_backward, embed_forward, embed_workspace_bytes  # noqa: E402
from tests.operator_util import U, Matrix, assert_within, half_step, stream, tiny, workspace  # noqa: E402


def _tokens(n, v, how, seed):
    g = torch.Generator().manual_seed(seed)
    if how == "uniform":
        return torch.randint(0, v, (n,), generator=g)
    if how == "same":
        return torch.full((n,), v // 2)
    if how == "half":                                       # half of the batch is one token
        t = torch.randint(0, v, (n,), generator=g)
        return torch.where(torch.rand(n, generator=g) < 0.5, torch.full_like(t, v - 1), t)
    if how == "outside":                                    # some on each side of the table
        return torch.randint(-3, v + 3, (n,), generator=g)
    if how == "none":
        return torch.full((n,), -1)
    u = torch.rand(n, generator=g, dtype=torch.float64)     # harmonic
    return (torch.exp(u * torch.log(torch.tensor(v + 1.0))) - 1).long().clamp(0, v - 1)


def _device(tok, bits):
    return tok.to(torch.int32 if bits == 32 else torch.int64).cuda()


def _backward(tok, v, w, kind="bf16", gkind="f32", pad=0, offset=0, bits=32, accumulate=False, factor=0.75, seed=0):
    n = tok.numel()
    g = torch.Generator().manual_seed(seed)
    DY = Matrix(n, w, kind, pad, offset, torch.randn((n, w), generator=g))
    old = torch.randn((v, w), generator=g)
    DT = Matrix(v, w, gkind, pad, offset, old if accumulate else None)
    before = DT.double() if accumulate else torch.zeros((v, w), dtype=torch.float64)
    t = _device(tok, bits)
    ws, room = workspace(embed_workspace_bytes(n, v, w))
    embed_backward(t.data_ptr() if n else 0, bits, n, DY.rows, v, w, factor, DT.rows, accumulate=accumulate, stream=stream(), **room)
    live = (tok >= 0) & (tok < v)
    at, dy = tok[live], DY.double()[live]
    want = torch.zeros((v, w), dtype=torch.float64).index_add_(0, at, dy) * factor
    size = torch.zeros((v, w), dtype=torch.float64).index_add_(0, at, dy.abs()) * abs(factor)
    count = torch.bincount(at, minlength=v)[:, None]
    want = want + before
    tol = (count + 10) * U * size + U * before.abs()
    got = DT.double()
    assert_within(got, want, tol + torch.where(count > 0, half_step(gkind) * (want.abs() + tol) + tiny(gkind), torch.zeros_like(tol)), "dtable")
    DT.check_guards()
    return DT


@pytest.mark.parametrize("n,v,w", [(1, 1, 1), (1, 1000, 64), (3, 5, 8), (31, 7, 33), (33, 100, 256), (64, 2, 257), (500, 50, 512), (2048, 3, 40),
                                   (2049, 4000, 24), (5000, 777, 130), (20000, 12, 16), (700, 30000, 96), (9000, 600000, 8)])
@pytest.mark.parametrize("how", ["uniform", "same", "half", "outside", "none", "harmonic"])
def test_gradient(n, v, w, how):
    _backward(_tokens(n, v, how, n + v), v, w)


@pytest.mark.parametrize("kind,gkind", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("f32", "bf16"), ("f16", "f32")])
@pytest.mark.parametrize("w,pad,offset", [(256, 0, 0), (264, 8, 8), (256, 1, 3), (100, 3, 1)])
def test_gradient_types_strides(kind, gkind, w, pad, offset):
    _backward(_tokens(900, 200, "half", 1), 200, w, kind, gkind, pad, offset, bits=64)


@pytest.mark.parametrize("gkind", ["f32", "bf16"])
@pytest.mark.parametrize("how", ["uniform", "half", "outside", "none"])
def test_gradient_accumulates(gkind, how):
    _backward(_tokens(1500, 400, how, 2), 400, 136, "bf16", gkind, accumulate=True)
    _backward(_tokens(1500, 400, how, 2), 400, 135, "bf16", gkind, accumulate=True)


def test_gradient_of_nothing():
    _backward(torch.zeros(0, dtype=torch.long), 50, 40)
    _backward(torch.zeros(0, dtype=torch.long), 50, 40, accumulate=True)


def test_same_bits_on_every_run():
    tok = _tokens(30000, 300, "harmonic", 5)
    assert torch.equal(_backward(tok, 300, 64).t, _backward(tok, 300, 64).t)


def test_tokens_of_64_bits_that_wrap_in_32():
    """a token of 2^32 + 1 is outside the table, not token 1"""
    tok = torch.tensor([1, (1 << 32) + 1, -(1 << 40), 2])
    _backward(tok, 4, 16, bits=64)
    T, Y = Matrix(4, 16, "f32", values=torch.arange(64.0).view(4, 16)), Matrix(4, 16, "f32")
    t = _device(tok, 64)
    embed_forward(t.data_ptr(), 64, 4, T.rows, 4, 16, 1.0, Y.rows, stream=stream())
    want = torch.zeros(4, 16)
    want[0], want[3] = T.t[1].cpu(), T.t[2].cpu()
    assert torch.equal(Y.t.cpu(), want)


@pytest.mark.parametrize("n,v,w,pad,offset", [(1, 1, 1, 0, 0), (5, 9, 8, 0, 0), (16, 1000, 4096, 0, 0), (333, 50, 1001, 0, 0), (70, 30, 2056, 8, 8), (70, 30, 256, 1, 1), (9, 4, 9000, 0, 0)])
@pytest.mark.parametrize("kind,ykind", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("bits", [32, 64])
def test_lookup(n, v, w, pad, offset, kind, ykind, bits):
    g = torch.Generator().manual_seed(n)
    tok = _tokens(n, v, "outside", n)
    T, Y = Matrix(v, w, kind, pad, offset, torch.randn((v, w), generator=g)), Matrix(n, w, ykind, pad, offset)
    t = _device(tok, bits)
    embed_forward(t.data_ptr(), bits, n, T.rows, v, w, 3.25, Y.rows, stream=stream())
    live = (tok >= 0) & (tok < v)
    want = torch.where(live[:, None], T.double()[tok.clamp(0, v - 1)] * 3.25, torch.zeros((), dtype=torch.float64))
    tol = U * want.abs()
    assert_within(Y.double(), want, tol + half_step(ykind) * (want.abs() + tol) + torch.where(live[:, None], tiny(ykind), 0.0), "y")
    Y.check_guards()


def test_lookup_in_no_table():
    t, Y = _device(torch.tensor([0, 1, -1]), 32), Matrix(3, 24, "f32")
    embed_forward(t.data_ptr(), 32, 3, Matrix(1, 24, "f32").rows, 0, 24, 1.0, Y.rows, stream=stream())
    assert bool((Y.t == 0).all())
