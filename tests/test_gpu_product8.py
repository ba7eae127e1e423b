"""Products of packed matrices against the sums in 64 bits.  Every scale and byte of a block differs, so a scale or element taken from
another place shows.

Tolerance: products are exact; a step of the tensor cores adds 32 of them to the accumulator and truncates each of the 33 summands at
2^-23 of the largest at most, so k / 32 steps are off by (k / 32) 33 2^-23 of the sum of absolute terms (a sum of fp32
multiply-adds by k 2^-24, which is less), shares of a split sum and the epilogue by a few 2^-24; one rounding to the type."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import matmul8, matmul8_workspace_bytes  # noqa: E402
from tests.operator_util import U, Matrix, PackedMatrix, assert_within, half_step, stream, tiny, unpack_reference, workspace  # noqa: E402


def _operand(n, k, seed, extra=0, spread=6):
    g = np.random.default_rng(seed)
    q = g.integers(0, 256, (n, k)).astype(np.uint8)
    q = np.where((q & 0x7f) == 0x7f, 0x38, q).astype(np.uint8)                        # no NaNs
    s = (127 + g.integers(-spread, spread + 1, (n, -(-k // 128)))).astype(np.uint8)
    # (what lies behind k and between rows would be NaN as an element or a scale)
    return PackedMatrix(n, k, extra, fill=0xff).put(q, s), torch.from_numpy(unpack_reference(q, s))


def _check(m, n, k, kind="f32", pad=0, offset=0, extra=0, seed=1):
    A, a = _operand(m, k, seed, extra)
    B, b = _operand(n, k, seed + 1, extra)
    scale = 2.0 ** -14 if kind == "f16" else 1.0                                      # (sums of up to 448^2 2^12 would overflow)
    if kind == "f16":
        A.s[:, :A.nb] -= 14
        a = a * scale
        B.s[:, :B.nb] -= 14
        b = b * scale
    Y = Matrix(m, n, kind, pad, offset)
    ws, room = workspace(matmul8_workspace_bytes(m, n, k))
    matmul8(A.packed, B.packed, m, n, k, Y.rows, stream=stream(), **room)
    a, b = a.cuda(), b.cuda()
    want, size = (a @ b.T).cpu(), (a.abs() @ b.abs().T).cpu()
    tol = (-(-k // 32) * 33 * 2 + 20) * U * size
    assert_within(Y.double(), want, tol + half_step(kind) * (want.abs() + tol) + tiny(kind), f"{m} x {n} x {k}")
    Y.check_guards()
    return Y


@pytest.mark.parametrize("m,n,k", [(128, 256, 128), (128, 256, 32), (128, 128, 512), (256, 256, 640), (300, 500, 1100), (129, 257, 129), (1500, 1333, 1100)])
def test_tiles(m, n, k):
    _check(m, n, k)


@pytest.mark.parametrize("m,n,k", [(5, 300, 700), (16, 1000, 4096), (32, 128, 64), (33, 4096, 512), (64, 200, 5000), (100, 513, 300), (128, 129, 128),
                                   (300, 5, 700), (1000, 17, 2000), (513, 100, 300), (5, 5, 5), (40, 40, 4000)])
def test_one_side_short(m, n, k):
    _check(m, n, k)


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 4096, 4096), (2, 4096, 4096), (3, 1000, 7001), (1, 30000, 800), (2, 33, 15), (3, 100, 1000), (4, 555, 513), (1000, 1, 777), (77, 3, 4097), (4, 4, 20000), (1, 3, 16)])
def test_few_rows(m, n, k):
    _check(m, n, k)


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("m,n,k,pad,offset,extra", [(200, 300, 400, 0, 0, 0), (130, 264, 200, 8, 8, 1), (130, 264, 200, 3, 1, 2), (20, 300, 400, 4, 0, 0), (3, 50, 60, 1, 1, 1), (150, 150, 9000, 2, 0, 0)])
def test_types_strides(kind, m, n, k, pad, offset, extra):
    _check(m, n, k, kind, pad, offset, extra)


@pytest.mark.parametrize("k", [1, 16, 31, 127, 128, 129, 511, 512, 513, 1024, 1025, 4224])
def test_lengths_of_k(k):
    _check(140, 270, k)
    _check(20, 270, k)


def test_many_tiles():
    """more tiles than SMs, ragged on both sides: the blocks walk, the scales' and the accumulator's buffers wrap"""
    _check(2500, 3333, 700, "bf16")
    _check(3000, 4111, 130, "bf16")


def test_scales_at_both_ends():
    """scales of 2^-110 and 2^110: the sum is of ordinary size"""
    q = np.full((160, 256), 0x38, np.uint8)                                           # ones
    A, B = PackedMatrix(160, 256).put(q, np.full((160, 2), 17, np.uint8)), PackedMatrix(160, 256).put(q, np.full((160, 2), 237, np.uint8))
    Y = Matrix(160, 160, "f32")
    ws, room = workspace(matmul8_workspace_bytes(160, 160, 256))
    matmul8(A.packed, B.packed, 160, 160, 256, Y.rows, stream=stream(), **room)
    assert bool((Y.t == 256.0).all())


@pytest.mark.parametrize("m", [2, 40, 200])
def test_nans_stay_in_their_row_and_column(m):
    n, k = 300, 500
    A, a = _operand(m, k, 5)
    B, b = _operand(n, k, 6)
    A.q[1, 70] = 0x7f
    B.q[5, 499] = 0xff
    Y = Matrix(m, n, "f32")
    ws, room = workspace(matmul8_workspace_bytes(m, n, k))
    matmul8(A.packed, B.packed, m, n, k, Y.rows, stream=stream(), **room)
    nan = torch.isnan(Y.t.cpu())
    want = torch.zeros(m, n, dtype=torch.bool)
    want[1], want[:, 5] = True, True
    assert torch.equal(nan, want)


def test_no_k_gives_zeros():
    Y = Matrix(7, 9, "bf16", pad=2)
    A, B = PackedMatrix(7, 0), PackedMatrix(9, 0)
    matmul8(A.packed, B.packed, 7, 9, 0, Y.rows, stream=stream())
    assert bool((Y.t == 0).all())
    Y.check_guards()


def test_same_bits_on_every_run():
    assert torch.equal(_check(300, 300, 3000, "f32").t, _check(300, 300, 3000, "f32").t)
