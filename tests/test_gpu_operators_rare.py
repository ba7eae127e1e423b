"""Rarely taken ways of the operators: infinities and NaNs in a row of the norm's and the lookup's gradient stay where the formula has
them, everything else keeps its bits; factors that are not finite; tables of millions of rows."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import (embed_backward, embed_forward, embed_workspace_bytes, layernorm_backward,  # noqa: E402
                                   layernorm_workspace_bytes, pack8)
from tests.operator_util import Matrix, PackedMatrix, stream, workspace  # noqa: E402

INF, NAN = float("inf"), float("nan")


# ---- gradient of the norm ----

class _Norm:
    def __init__(self, n, width, kind, pad, packed):
        g = torch.Generator().manual_seed(n + width)
        r = lambda *s: torch.randn(s, generator=g)
        self.n, self.width, self.packed, self.kind, self.pad = n, width, packed, kind, pad
        self.X, self.DY = Matrix(n, width, kind, pad, 0, r(n, width)), Matrix(n, width, kind, pad, 0, r(n, width))
        self.W = Matrix(1, width, "f32", values=1 + 0.1 * r(1, width))
        x = self.X.t.float()
        self.mean, self.rstd = x.mean(1), torch.rsqrt(x.var(1, unbiased=False) + 1e-5)

    def run(self):
        n, width = self.n, self.width
        DX, DW, DB = Matrix(n, width, self.kind, self.pad), Matrix(1, width, "f32"), Matrix(1, width, "f32")
        K = None
        if self.packed:
            K = PackedMatrix(n, width, fill=0xff)
            pack8(self.X.rows, n, width, K.packed, stream=stream())
        ws, room = workspace(layernorm_workspace_bytes(n, width))
        layernorm_backward(self.DY.rows, None if K else self.X.rows, K.packed if K else None, n, width, self.mean.data_ptr(), self.rstd.data_ptr(), DX.rows,
                           self.W.rows, DW.rows, DB.rows, stream=stream(), **room)
        return DX.t.cpu(), DW.t[0].cpu(), DB.t[0].cpu()


# (a warp a row, groups, clusters, long rows; aligned and not)
@pytest.mark.parametrize("n,width,pad", [(40, 96, 0), (40, 96, 1), (200, 1024, 0), (200, 1001, 0), (30, 4104, 0), (30, 8200, 0), (30, 9001, 0), (9, 33000, 0)])
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("where", ["dy", "x", "mean", "rstd"])
def test_gradient_of_the_norm_beside_rows_that_are_not_finite(n, width, pad, packed, where):
    s = _Norm(n, width, "bf16", pad, packed)
    dx, dw, db = s.run()
    rows, columns = torch.tensor([0, n // 2, n - 1]), torch.tensor([0, width // 3, width - 1])
    values = torch.tensor([NAN, INF, -INF], device="cuda")
    if where in ("dy", "x"):
        (s.DY if where == "dy" else s.X).t[rows.cuda(), columns.cuda()] = values.bfloat16()
    else:
        getattr(s, where)[rows.cuda()] = values
    bx, bw, bb = s.run()
    other = torch.ones(n, dtype=torch.bool)
    other[rows] = False
    assert torch.equal(bx[other], dx[other]) and bool(torch.isfinite(dx).all())
    assert not bool(torch.isfinite(bx[rows]).any())
    hit = torch.zeros(width, dtype=torch.bool)
    hit[columns] = True
    if packed and where == "x":
        # (the block of an infinity has another scale where that was its largest element: its columns may change)
        near = torch.zeros(width, dtype=torch.bool)
        for c in columns:
            near[int(c) // 128 * 128:int(c) // 128 * 128 + 128] = True
        assert torch.equal(bw[~near], dw[~near]) and not bool(torch.isfinite(bw[hit]).any()) and torch.equal(bb, db)
    elif where in ("dy", "x"):
        assert torch.equal(bw[~hit], dw[~hit]) and not bool(torch.isfinite(bw[hit]).any())
        assert torch.equal(bb[~hit], db[~hit]) and (where == "x" or not bool(torch.isfinite(bb[hit]).any())) and (where == "dy" or torch.equal(bb, db))
    else:
        assert not bool(torch.isfinite(bw).any()) and torch.equal(bb, db)


# ---- lookup and its gradient ----

def _gradient(tok, DY, v, width, factor=0.5, kind="f32", accumulate=None):
    DT = Matrix(v, width, kind, values=accumulate)
    if accumulate is None:
        DT.t.fill_(NAN)
    ws, room = workspace(embed_workspace_bytes(tok.numel(), v, width))
    embed_backward(tok.data_ptr(), tok.element_size() * 8, tok.numel(), DY.rows, v, width, factor, DT.rows, accumulate=accumulate is not None, stream=stream(), **room)
    DT.check_guards()
    return DT.t


@pytest.mark.parametrize("width", [40, 300, 301])
@pytest.mark.parametrize("n,v", [(200, 30), (5000, 30), (3000, 2000)])
def test_gradient_of_the_lookup_beside_rows_that_are_not_finite(n, v, width):
    g = torch.Generator().manual_seed(n)
    tok = torch.randint(-2, v + 2, (n,), generator=g)
    tok[n // 2] = v // 2
    tok[::7] = -1                                                  # padding: what its rows of dy hold counts for nothing
    t = tok.int().cuda()
    DY = Matrix(n, width, "bf16", values=torch.randn((n, width), generator=g))
    want = _gradient(t, DY, v, width)
    at = n // 2 if tok[n // 2] >= 0 else n // 2 + 1
    row, column = int(tok[at]), width // 2
    DY.t[torch.arange(0, n, 7).cuda()] = NAN
    inside = 0 <= row < v
    DY.t[at, column] = NAN
    got = _gradient(t, DY, v, width)
    hit = torch.zeros((v, width), dtype=torch.bool, device="cuda")
    if inside:
        hit[row, column] = True
    assert torch.equal(got[~hit], want[~hit]) and bool(torch.isnan(got[hit]).all()) and bool(torch.isfinite(want).all())


@pytest.mark.parametrize("factor", [INF, -INF, NAN, 0.0])
@pytest.mark.parametrize("width", [64, 65])
def test_factors(factor, width):
    """padding and rows without tokens are zeros whatever the factor"""
    n, v = 50, 90
    tok = torch.arange(n) % 20
    tok[5], tok[6] = -1, v
    t = tok.int().cuda()
    ones = torch.ones((v, width))
    T, Y, DY = Matrix(v, width, "f32", values=ones), Matrix(n, width, "f32"), Matrix(n, width, "f32", values=ones[:n])
    embed_forward(t.data_ptr(), 32, n, T.rows, v, width, factor, Y.rows, stream=stream())
    live = (tok >= 0) & (tok < v)
    want = torch.where(live[:, None], torch.full((n, width), factor), torch.zeros(()))
    assert torch.equal(torch.nan_to_num(Y.t.cpu(), nan=7.0), torch.nan_to_num(want, nan=7.0))
    count = torch.bincount(tok[live], minlength=v)[:, None]
    want = torch.where(count > 0, count * factor, torch.zeros(())).expand(v, width)
    assert torch.equal(torch.nan_to_num(_gradient(t, DY, v, width, factor).cpu(), nan=7.0), torch.nan_to_num(want, nan=7.0))


@pytest.mark.parametrize("v,width,bits", [(5_000_000, 8, 32), (4_700_003, 3, 64), ((1 << 27) + 5, 1, 32), ((1 << 27) + 5, 1, 64)])
@pytest.mark.parametrize("n", [70, 6000])
def test_tables_of_millions_of_rows(v, width, bits, n):
    """more rows a block than it notes at a time; keys of four digits.  Whole numbers: the sums are exact"""
    g = torch.Generator().manual_seed(v % 97)
    tok = torch.randint(0, v, (n,), generator=g)
    tok[: n // 3] = tok[n // 2]                                    # a row of many
    tok[1], tok[2], tok[3], tok[4] = 0, v - 1, -1, v
    t = tok.to(torch.int32 if bits == 32 else torch.int64).cuda()
    dy = torch.randint(-4, 5, (n, width), generator=g).float()
    DY = Matrix(n, width, "bf16", values=dy)
    live = (tok >= 0) & (tok < v)
    want = torch.zeros((v, width), device="cuda").index_add_(0, tok[live].cuda(), dy[live].cuda())
    assert torch.equal(_gradient(t, DY, v, width, 1.0), want)
    assert torch.equal(_gradient(t, DY, v, width, 1.0, accumulate=torch.ones((), device="cuda").expand(v, width)), want + 1)
    torch.cuda.empty_cache()
