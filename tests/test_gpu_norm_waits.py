"""Waits of the layer norm's kernels that run out: what they were for is NaN, in every output, nothing else is touched, and the next call is as
if nothing had been.  The waits count as run out from the start here; no data is missing, so the kernels' own waits for what is still
on its way all end."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import (debug_lost_waits, layernorm_backward, layernorm_forward, layernorm_workspace_bytes)  # noqa: E402
from tests.operator_util import Matrix, PackedMatrix, pack_reference, same_codes, stream, workspace  # noqa: E402


def _run(x, dy, w, kind, pad, packed):
    n, width = x.shape
    X, DY, Y, DX = (Matrix(n, width, kind, pad, 0, v) for v in (x, dy, None, None))
    W, DW, DB = Matrix(1, width, "f32", values=w), Matrix(1, width, "f32"), Matrix(1, width, "f32")
    K = PackedMatrix(n, width)
    mean, rstd = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    layernorm_forward(X.rows, n, width, Y.rows, W.rows, None, 1e-5, mean.data_ptr(), rstd.data_ptr(), K.packed if packed else None, stream=stream())
    fm, fr = X.t.float().mean(1), torch.rsqrt(X.t.float().var(1, unbiased=False) + 1e-5)
    if packed:
        # (a good checkpoint for the backward pass)
        q, s = pack_reference(X.double().numpy())
        G = PackedMatrix(n, width).put(q, s)
    ws, room = workspace(layernorm_workspace_bytes(n, width))
    layernorm_backward(DY.rows, None if packed else X.rows, G.packed if packed else None, n, width, fm.data_ptr(), fr.data_ptr(), DX.rows, W.rows, DW.rows, DB.rows,
                       stream=stream(), **room)
    torch.cuda.synchronize()
    for m in (Y, DX, DW, DB, K):
        m.check_guards()
    return dict(y=Y.t.cpu(), mean=mean.cpu(), rstd=rstd.cpu(), dx=DX.t.cpu(), dw=DW.t.cpu(), db=DB.t.cpu()), K.bytes() if packed else None


# a warp a row, groups, clusters: rows come by copies.  Off every boundary: clusters wait for each other only
@pytest.mark.parametrize("n,width,pad", [(1500, 96, 0), (1000, 1024, 0), (2500, 4096, 0), (300, 8200, 0), (300, 20000, 0), (400, 8192, 0), (1200, 1001, 0), (300, 9001, 0)])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("packed", [False, True])
def test_waits_that_run_out(n, width, pad, kind, packed):
    g = torch.Generator().manual_seed(width)
    x, dy, w = torch.randn((n, width), generator=g), torch.randn((n, width), generator=g), torch.ones((1, width))
    want, kept = _run(x, dy, w, kind, pad, packed)
    assert all(bool(torch.isfinite(t).all()) for t in want.values())
    debug_lost_waits(True)
    try:
        got, codes = _run(x, dy, w, kind, pad, packed)
    finally:
        debug_lost_waits(False)
    copies, clusters = width % 8 == 0, width > 4096
    # (the forward kernel by groups of a large block has no such switch)
    large = clusters and n >= 296 and width <= (13312 if kind == "f32" else 18432) and not (packed and kind == "f32")
    for name, t in got.items():
        if copies and large and name in ("y", "mean", "rstd"):
            assert torch.equal(t, want[name]), name
        elif copies or (clusters and name not in ("dw", "db")):
            assert bool(torch.isnan(t).all()), name
        else:
            assert torch.equal(t, want[name]), name
    if packed:
        # (fp32 rows are packed by the pass itself, others by a kernel that waits for nothing)
        if kind == "f32" and copies:
            assert bool(((codes[0] & 0x7f) == 0x7f).all())
        else:
            assert same_codes(codes[0], kept[0]) and np.array_equal(codes[1], kept[1])
    again, codes = _run(x, dy, w, kind, pad, packed)
    assert all(torch.equal(again[name], want[name]) for name in want) and (not packed or same_codes(codes[0], kept[0]))
