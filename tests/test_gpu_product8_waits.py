"""A product whose wait for operands runs out: every output is NaN (no part of a sum passes for the sum), nothing else is written, and the
next call is as if nothing had been.  A wait for each tile's operands counts as run out here, behind the last of its multiplications; all operands
come, so what the kernel still waits for in the end does too."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import debug_lost_waits, matmul8, matmul8_workspace_bytes  # noqa: E402
from tests.operator_util import Matrix, PackedMatrix, stream, workspace  # noqa: E402


def _operand(n, k, seed):
    g = np.random.default_rng(seed)
    q = g.integers(0, 256, (n, k)).astype(np.uint8)
    q = np.where((q & 0x7f) == 0x7f, 0x38, q).astype(np.uint8)
    return PackedMatrix(n, k, fill=0xff).put(q, (127 + g.integers(-3, 4, (n, -(-k // 128)))).astype(np.uint8))


def _run(A, B, m, n, k, kind):
    Y = Matrix(m, n, kind, pad=3)
    ws, room = workspace(matmul8_workspace_bytes(m, n, k))
    matmul8(A.packed, B.packed, m, n, k, Y.rows, stream=stream(), **room)
    torch.cuda.synchronize()
    Y.check_guards()
    return Y.t.cpu()


# one block of k and many, tiles of every width, k in shares, more tiles than blocks; pairs of blocks
@pytest.mark.parametrize("m,n,k", [(128, 129, 100), (20, 300, 4000), (1000, 60, 700), (300, 120, 1100), (300, 500, 3000), (2500, 3333, 700)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_a_wait_that_runs_out(m, n, k, kind):
    A, B = _operand(m, k, 1), _operand(n, k, 2)
    want = _run(A, B, m, n, k, kind)
    assert bool(torch.isfinite(want).all())
    debug_lost_waits(True)
    try:
        got = _run(A, B, m, n, k, kind)
    finally:
        debug_lost_waits(False)
    assert bool(torch.isnan(got).all())
    assert torch.equal(_run(A, B, m, n, k, kind), want)
