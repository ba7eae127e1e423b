"""Matrices in 8 bits: bytes and scales equal the definition bit by bit, from every type, alignment and width; the transpose; values
come back exactly; infinities, NaNs, zeros, the smallest and the largest numbers."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import pack8, repack8, unpack8  # noqa: E402
from tests.operator_util import (Matrix, PackedMatrix, half_step, pack_reference, same_codes, stream, tiny,  # noqa: E402
                                 unpack_reference)

SHAPES = [(1, 1), (1, 7), (3, 8), (5, 127), (2, 128), (7, 129), (1, 1000), (33, 260), (130, 1537), (4, 4096), (65, 2049), (1000, 3)]


def _values(n, w, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, w), generator=g) * torch.exp(3 * torch.randn((n, 1), generator=g))
    # ties and borders: halves of e4m3 steps, amounts at 448 times a power of two and the next number
    x[0, 0] = 448.0
    if w > 4:
        x[0, 1:5] = torch.tensor([17.0, -19.0, 2.0 ** -10, 3 * 2.0 ** -10])
    if n > 2:
        x[1] = 0.0
        x[2] = torch.nextafter(torch.tensor(448.0), torch.tensor(500.0)) * 2.0 ** -20
    return x


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,w", SHAPES)
@pytest.mark.parametrize("pad,offset", [(0, 0), (3, 1), (8, 0)])
def test_pack_and_back(kind, n, w, pad, offset):
    x = Matrix(n, w, kind, pad, offset, _values(n, w, n * w).clamp(-60000, 60000))
    p = PackedMatrix(n, w, extra=pad % 2)
    pack8(x.rows, n, w, p.packed, stream=stream())
    q, s = p.bytes()
    wq, ws = pack_reference(x.double().numpy())
    assert np.array_equal(s, ws) and same_codes(q, wq)
    p.check_guards()
    y = Matrix(n, w, kind, pad, offset)
    unpack8(p.packed, n, w, y.rows, stream=stream())
    back = torch.from_numpy(unpack_reference(q, s)).to(x.t.dtype)           # rounded once (exactly, but for fp16's subnormal numbers)
    assert bool((y.t.cpu() == back).all())
    y.check_guards()
    want = x.double()
    assert bool(((y.double() - want).abs() <= 2.0 ** -4 * want.abs() + torch.from_numpy(np.repeat(2.0 ** (s.astype(float) - 137), 128, 1)[:, :w]) + tiny(kind) + half_step(kind) * want.abs()).all())


@pytest.mark.parametrize("n,w", SHAPES + [(128, 128), (127, 300), (129, 257), (1025, 40), (16, 1), (256, 384)])
def test_transpose(n, w):
    q, s = pack_reference(_values(n, w, 7 * n + w).double().numpy())
    a, b = PackedMatrix(n, w, extra=1, fill=0x7f).put(q, s), PackedMatrix(w, n, extra=1)      # (NaNs between the rows must not be read as elements)
    repack8(a.packed, n, w, b.packed, stream=stream())
    wq, ws = pack_reference(unpack_reference(q, s).T)
    gq, gs = b.bytes()
    assert np.array_equal(gs, ws) and same_codes(gq, wq)
    b.check_guards()


@pytest.mark.parametrize("offset", [0, 1])
def test_special_values(offset):
    x = torch.ones((6, 300))
    x[0, :3] = torch.tensor([float("inf"), -float("inf"), float("nan")])       # do not count for the scale
    x[1] = float("nan")
    x[2] = 0.0
    x[2, 5] = -0.0
    x[3] = 1e-45                                                               # subnormal: the least scale
    x[4] = torch.finfo(torch.float32).max
    x[5, 1] = 2.0 ** -126
    m, p = Matrix(6, 300, "f32", 0, offset, x), PackedMatrix(6, 300)
    pack8(m.rows, 6, 300, p.packed, stream=stream())
    q, s = p.bytes()
    wq, ws = pack_reference(x.double().numpy())
    assert np.array_equal(s, ws) and same_codes(q, wq)
    y = Matrix(6, 300, "f32")
    unpack8(p.packed, 6, 300, y.rows, stream=stream())
    # the largest fp32 rounds to 256 2^120, which is an infinity in fp32: values are those of the type that is written or read
    with np.errstate(over="ignore"):
        back = unpack_reference(q, s).astype(np.float32)
    assert np.isposinf(back[4]).all()
    np.testing.assert_array_equal(y.t.cpu().numpy(), back)
    t = PackedMatrix(300, 6)
    repack8(p.packed, 6, 300, t.packed, stream=stream())
    wq, ws = pack_reference(back.T)
    gq, gs = t.bytes()
    assert np.array_equal(gs, ws) and same_codes(gq, wq)


def test_every_byte_comes_back():
    """all 256 codes under scales of every size, the largest overflow fp32 (2^127 448), the smallest are subnormal"""
    q = np.tile(np.arange(256, dtype=np.uint8), (7, 1))
    s = np.array([[0, 1], [1, 0], [10, 20], [127, 128], [247, 200], [254, 3], [255, 127]], np.uint8)
    p, y = PackedMatrix(7, 256).put(q, s), Matrix(7, 256, "f32")
    unpack8(p.packed, 7, 256, y.rows, stream=stream())
    with np.errstate(over="ignore"):
        want = unpack_reference(q, s).astype(np.float32)
    np.testing.assert_array_equal(y.t.cpu().numpy(), want)


def test_many_rows_offsets_beyond_32_bits():
    """rows whose byte offsets pass 2^32: a stride, not the data, makes them far"""
    n, w, stride = 5, 256, 1 << 31
    buf = torch.zeros(4 * stride + w, dtype=torch.uint8, device="cuda")
    rows = torch.as_strided(buf, (n, w), (stride, 1))
    q, s = pack_reference(_values(n, w, 3).double().numpy())
    rows.copy_(torch.from_numpy(q))
    sc = PackedMatrix(n, w).put(q, s)
    from paper_1711_01348_b200 import Packed
    far = Packed(buf.data_ptr(), sc.s.data_ptr(), stride, sc.ss)
    y = Matrix(n, w, "f32")
    # (the last row of a packed matrix has the length of the others: read all but it)
    unpack8(far, n - 1, w, y.rows, stream=stream())
    np.testing.assert_array_equal(y.double().numpy()[:n - 1], unpack_reference(q, s)[:n - 1])
