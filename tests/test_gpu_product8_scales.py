"""Products of packed matrices whose scales are far from one: large on one side and small on the other, so that the sum is of ordinary
size although no partial product with one of the scales alone would be; results near both ends of fp32; scales that stand for NaN.

Tolerance: as in test_gpu_product8.py, and 2^-150 for every rounding to a subnormal number (one a piece of sixteen, sixteen joined)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import matmul8, matmul8_workspace_bytes, pack8  # noqa: E402
from tests.operator_util import U, Matrix, PackedMatrix, assert_within, half_step, stream, unpack_reference, workspace  # noqa: E402


def _operand(n, k, byte, seed, positive=False):
    """random codes, scales within two of `byte`"""
    g = np.random.default_rng(seed)
    q = g.integers(0, 256, (n, k)).astype(np.uint8)
    q = np.where((q & 0x7f) == 0x7f, 0x7e, q).astype(np.uint8)                        # 448 in the place of NaNs
    if positive:
        q &= 0x7f
    s = np.clip(byte + g.integers(-2, 3, (n, -(-k // 128))), 0, 254).astype(np.uint8)
    return PackedMatrix(n, k, fill=0xff).put(q, s), torch.from_numpy(unpack_reference(q, s))


def _product(A, B, m, n, k, kind="f32"):
    Y = Matrix(m, n, kind)
    ws, room = workspace(matmul8_workspace_bytes(m, n, k))
    matmul8(A.packed, B.packed, m, n, k, Y.rows, stream=stream(), **room)
    Y.check_guards()
    return Y.double()


def _check(A, a, B, b, m, n, k, kind="f32"):
    want, size = a @ b.T, a.abs() @ b.abs().T
    tol = (-(-k // 32) * 33 * 2 + 20) * U * size + (-(-k // 16) + 16) * 2.0 ** -150
    assert_within(_product(A, B, m, n, k, kind), want, tol + (half_step(kind) if kind != "f32" else 0) * (want.abs() + tol), f"{m} x {n} x {k}")


# bytes of the scales: their powers add up to 0, to +-25, to the ends of the range
PAIRS = [(240, 14), (14, 240), (254, 0), (0, 254), (247, 7), (200, 79), (60, 169), (227, 50)]


@pytest.mark.parametrize("sa,sb", PAIRS)
@pytest.mark.parametrize("few", [1, 2, 3, 4])
def test_few_rows(few, sa, sb):
    for m, n, k in ((few, 50, 700), (50, few, 700), (few, 9, 17), (few, 4, 1)):
        A, a = _operand(m, k, sa, m + n)
        B, b = _operand(n, k, sb, m + 2 * n)
        _check(A, a, B, b, m, n, k)
        _check(A, a, B, b, m, n, k, "bf16")


@pytest.mark.parametrize("sa,sb", PAIRS)
@pytest.mark.parametrize("m,n,k", [(160, 160, 256), (16, 300, 700), (300, 20, 1100), (300, 300, 300)])
def test_tiles(m, n, k, sa, sb):
    A, a = _operand(m, k, sa, m + n)
    B, b = _operand(n, k, sb, m + 2 * n)
    _check(A, a, B, b, m, n, k)


@pytest.mark.parametrize("few", [1, 2, 3, 4])
@pytest.mark.parametrize("way", [0, 1])
@pytest.mark.parametrize("large,small", [(1e35, 1e-30), (1e38, 1e-36), (1e36, 1e-36)])
def test_few_rows_of_packed_numbers(few, way, large, small):
    g = torch.Generator().manual_seed(few)
    m, n, k = (few, 37, 900) if way else (37, few, 900)
    ms, ns = (large, small) if few % 2 else (small, large)
    x, y = torch.rand((m, k), generator=g).add(1.0).mul(ms), torch.randn((n, k), generator=g).clamp(-3, 3).mul(ns)
    X, Y, A, B = Matrix(m, k, "f32", values=x), Matrix(n, k, "f32", values=y), PackedMatrix(m, k), PackedMatrix(n, k)
    pack8(X.rows, m, k, A.packed, stream=stream())
    pack8(Y.rows, n, k, B.packed, stream=stream())
    _check(A, torch.from_numpy(unpack_reference(*A.bytes())), B, torch.from_numpy(unpack_reference(*B.bytes())), m, n, k)


@pytest.mark.parametrize("few", [1, 2, 3, 4])
@pytest.mark.parametrize("sa,sb", [(60, 60), (2, 115), (110, 4), (30, 80)])
def test_few_rows_with_results_near_the_smallest(few, sa, sb):
    """products of scales from 2^-134 to 2^-144: pieces of a sum are subnormal numbers"""
    A, a = _operand(few, 300, sa, 1)
    B, b = _operand(30, 300, sb, 2)
    _check(A, a, B, b, few, 30, 300)


@pytest.mark.parametrize("few", [1, 2, 3, 4])
def test_few_rows_beyond_the_ends(few):
    n, k = 20, 300
    for sa, sb, want in ((240, 240, float("inf")), (254, 254, float("inf")), (20, 20, 0.0), (0, 0, 0.0), (130, 250, float("inf"))):
        A, a = _operand(few, k, sa, 3, positive=True)
        B, b = _operand(n, k, sb, 4, positive=True)
        assert bool((_product(A, B, few, n, k) == want).all())


@pytest.mark.parametrize("few", [1, 2, 3, 4])
def test_few_rows_with_scales_that_stand_for_nan(few):
    """such a block is NaN whatever its elements, zeros too, and whatever the other side's scale"""
    n, k = 33, 500
    A, a = _operand(few, k, 127, 5)
    B, b = _operand(n, k, 127, 6)
    B.q[5] = 0
    B.s[5, 1], B.s[9, 3] = 255, 255
    A.s[few - 1, 2] = 0
    B.s[9, 2] = 0
    for way in range(2):
        y = _product(A, B, few, n, k) if way == 0 else _product(B, A, n, few, k).T
        want = torch.zeros(few, n, dtype=torch.bool)
        want[:, 5], want[:, 9] = True, True
        assert torch.equal(torch.isnan(y), want)
    A.s[0, 3] = 255
    want[0] = True
    assert torch.equal(torch.isnan(_product(A, B, few, n, k)), want)
