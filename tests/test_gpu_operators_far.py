"""Rows far apart: offsets beyond 2^31 elements and 2^32 bytes in every operator.  A stride, not the data, makes them far; what is written
equals, bit by bit, what the same call gives with the rows next to each other."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import (Packed, Rows, embed_backward, embed_forward, embed_workspace_bytes, layernorm_backward,  # noqa: E402
                                   layernorm_forward, layernorm_workspace_bytes, matmul8, matmul8_workspace_bytes, pack8, repack8, unpack8)
from tests.operator_util import GUARD, TYPES, stream, workspace  # noqa: E402

FAR = (1 << 30) + 64                # elements between rows: the fourth row is beyond 2^31 elements, of 16 bits beyond 2^32 bytes


@pytest.fixture(autouse=True)
def _give_memory_back():
    yield
    torch.cuda.synchronize()
    torch.cuda.empty_cache()


class _Matrix:
    def __init__(self, n, width, kind, stride, offset=0, values=None):
        self.n, self.width = n, width
        self.buf = torch.empty(offset + (n - 1) * stride + width + 64, dtype=TYPES[kind], device="cuda")
        # the rows and up to 32 elements behind each of them
        self.around = torch.as_strided(self.buf, (n, width + min(32, stride - width)), (stride, 1), offset)
        self.around.fill_(GUARD)
        self.t = self.around[:, :width]
        if values is not None:
            self.t.copy_(values)
        self.rows = Rows(self.buf.data_ptr() + offset * self.buf.element_size(), stride, kind)

    def get(self):
        torch.cuda.synchronize()
        assert bool((self.around[:, self.width:] == GUARD).all()), "written behind a row"
        return self.t.cpu()


class _Packed:
    """every row has the length of the stride, the last one too"""

    def __init__(self, n, width, stride=0, scale_stride=0):
        self.n, self.width, self.nb = n, width, -(-width // 128)
        qs, ss = stride or -(-width // 16) * 16, scale_stride or -(-self.nb // 4) * 4
        self.qbuf, self.sbuf = torch.empty(n * qs, dtype=torch.uint8, device="cuda"), torch.empty(n * ss, dtype=torch.uint8, device="cuda")
        self.q, self.s = torch.as_strided(self.qbuf, (n, -(-width // 16) * 16), (qs, 1)), torch.as_strided(self.sbuf, (n, -(-self.nb // 4) * 4), (ss, 1))
        self.q.fill_(0x7f)
        self.s.fill_(255)
        self.packed = Packed(self.qbuf.data_ptr(), self.sbuf.data_ptr(), qs, ss)

    def put(self, other):
        self.q[:, :self.width] = other.q[:, :self.width]
        self.s[:, :self.nb] = other.s[:, :self.nb]
        return self

    def get(self):
        torch.cuda.synchronize()
        return self.q[:, :self.width].cpu(), self.s[:, :self.nb].cpu()


def _random(n, w, seed):
    return torch.randn((n, w), generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("width,offset", [(64, 0), (65, 1), (1200, 0)])
def test_lookup(width, offset):
    n, v = 5, 4
    tok = torch.tensor([3, 0, 2, 1, 3], dtype=torch.int32, device="cuda")
    out = []
    for stride in (width + 8, FAR):
        T, Y = _Matrix(v, width, "bf16", stride, offset, _random(v, width, 1)), _Matrix(n, width, "bf16", stride, offset)
        embed_forward(tok.data_ptr(), 32, n, T.rows, v, width, 2.5, Y.rows, stream=stream())
        out.append(Y.get())
    assert torch.equal(*out)


@pytest.mark.parametrize("width,offset", [(64, 0), (65, 1), (1200, 0)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_gradient_of_the_lookup(width, offset, accumulate):
    n, v = 5, 4
    tok = torch.tensor([3, 0, 3, 1, 3], dtype=torch.int32, device="cuda")           # row 2 has none
    out = []
    for stride in (width + 8, FAR):
        DY, DT = _Matrix(n, width, "bf16", stride, offset, _random(n, width, 1)), _Matrix(v, width, "bf16", stride, offset, _random(v, width, 2))
        ws, room = workspace(embed_workspace_bytes(n, v, width))
        embed_backward(tok.data_ptr(), 32, n, DY.rows, v, width, 2.5, DT.rows, accumulate=accumulate, stream=stream(), **room)
        out.append(DT.get())
    assert torch.equal(*out)
    assert accumulate or bool((out[0][2] == 0).all())


# a warp a row, groups, clusters, rows of any length; rows off every boundary; many wide rows (groups of a large block)
@pytest.mark.parametrize("n,width,offset,stride", [(4, 96, 0, FAR), (4, 1024, 0, FAR), (4, 1001, 1, FAR), (4, 8200, 0, FAR), (4, 9001, 1, FAR), (4, 33000, 0, FAR),
                                                   (300, 5000, 0, (1 << 23) + 64)])
@pytest.mark.parametrize("eight", [False, True])
def test_norm(n, width, offset, stride, eight):
    x, dy, w, b = _random(n, width, 1), _random(n, width, 2), 1 + 0.1 * _random(1, width, 3), _random(1, width, 4)
    out = []
    for st in (-(-width // 8) * 8 + 8, stride):
        X, DY, Y, DX = (_Matrix(n, width, "bf16", st, offset, v) for v in (x, dy, None, None))
        W, B, DW, DB = (_Matrix(1, width, "f32", width, 0, v) for v in (w, b, None, None))
        far = st == stride
        K = _Packed(n, width, st // 16 * 16 if far else 0, 1 << 23 if far and n > 4 else FAR if far else 0) if eight else None
        mean, rstd = (torch.empty(n, device="cuda") for _ in range(2))
        layernorm_forward(X.rows, n, width, Y.rows, W.rows, B.rows, 1e-5, mean.data_ptr(), rstd.data_ptr(), K.packed if K else None, stream=stream())
        ws, room = workspace(layernorm_workspace_bytes(n, width))
        layernorm_backward(DY.rows, None if K else X.rows, K.packed if K else None, n, width, mean.data_ptr(), rstd.data_ptr(), DX.rows, W.rows, DW.rows, DB.rows,
                           stream=stream(), **room)
        out.append([Y.get(), DX.get(), DW.get(), DB.get(), mean.cpu(), rstd.cpu(), *(K.get() if K else ())])
        del X, DY, Y, DX, K
    assert all(torch.equal(s, t) for s, t in zip(*out))
    assert all(bool(torch.isfinite(t).all()) for t in out[0][:6])


def test_checkpoint_in_the_pass_of_the_norm():
    """fp32 rows"""
    n, width, out = 4, 1024, []
    for st, far in ((width, 0), (FAR, FAR)):
        X, Y, K = _Matrix(n, width, "f32", st, 0, _random(n, width, 1)), _Matrix(n, width, "f32", st), _Packed(n, width, far, far)
        layernorm_forward(X.rows, n, width, Y.rows, checkpoint=K.packed, stream=stream())
        out.append([Y.get(), *K.get()])
    assert all(torch.equal(s, t) for s, t in zip(*out))


@pytest.mark.parametrize("kind,width,offset", [("bf16", 1000, 0), ("bf16", 1000, 1), ("f32", 700, 0), ("f32", 700, 1)])
def test_packing(kind, width, offset):
    n, out = 4, []
    for far in (0, FAR):
        st = far or -(-width // 8) * 8
        X, K, Y = _Matrix(n, width, kind, st, offset, _random(n, width, 1)), _Packed(n, width, far, far), _Matrix(n, width, kind, st, offset)
        pack8(X.rows, n, width, K.packed, stream=stream())
        unpack8(K.packed, n, width, Y.rows, stream=stream())
        out.append([Y.get(), *K.get()])
    assert all(torch.equal(s, t) for s, t in zip(*out))


@pytest.mark.parametrize("n,width", [(4, 300), (300, 4)])
def test_transpose(n, width):
    """rows far apart on the side that has few of them"""
    X, near = _Matrix(n, width, "f32", width, 0, _random(n, width, 1)), _Packed(n, width)
    pack8(X.rows, n, width, near.packed, stream=stream())
    out = []
    for far in (0, FAR):
        K, T = _Packed(n, width, far if n == 4 else 0, far if n == 4 else 0).put(near), _Packed(width, n, far if n != 4 else 0, far if n != 4 else 0)
        repack8(K.packed, n, width, T.packed, stream=stream())
        out.append(T.get())
    assert all(torch.equal(s, t) for s, t in zip(*out))


# few rows; tiles with either operand along the lanes, a split sum, pairs of blocks
@pytest.mark.parametrize("m,n,k,far", [(3, 200, 300, 1 << 25), (160, 200, 300, 1 << 25), (20, 200, 1500, 1 << 25), (2400, 2050, 200, 1 << 21)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_product(m, n, k, far, kind):
    near = []
    for rows, seed in ((m, 1), (n, 2)):
        X, K = _Matrix(rows, k, "f32", k, 0, _random(rows, k, seed)), _Packed(rows, k)
        pack8(X.rows, rows, k, K.packed, stream=stream())
        near.append(K)
    out = []
    for st in (0, far):
        A, B = (_Packed(K.n, k, st, st).put(K) for K in near)
        # (the rows of y are as far apart as makes the last one pass 2^31 elements)
        Y = _Matrix(m, n, kind, max(n, (1 << 31) // (m - 1) + 64 & ~63) if st else -(-n // 32) * 32)
        ws, room = workspace(matmul8_workspace_bytes(m, n, k))
        matmul8(A.packed, B.packed, m, n, k, Y.rows, stream=stream(), **room)
        out.append(Y.get())
        del A, B, Y
    assert torch.equal(*out) and bool(torch.isfinite(out[0]).all())
