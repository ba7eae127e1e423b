"""Layer norm against its formula in 64 bits: every type, odd widths, strides and offsets, both sides of each change of kernel
(512 columns a warp, 4096 or 8192 a block, 32768 a cluster), few and many rows, from x and from its 8-bit form.

Tolerances: u = 2^-24 is the rounding of an operation, a sum over a row passes at most depth(width) of them (16 elements or
width / 1024 a thread, ten levels of shuffles), a result is rounded to its type once."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import layernorm_backward, layernorm_forward, layernorm_workspace_bytes  # noqa: E402
from tests.operator_util import (U, Matrix, PackedMatrix, assert_within, half_step, pack_reference, same_codes, stream,  # noqa: E402
                                 tiny, unpack_reference, workspace)

# (either side of a warp, a block, clusters of 2, 4 and 8 blocks of either pass, and of the longest row that a cluster holds)
WIDTHS = [1, 2, 7, 8, 33, 128, 500, 512, 513, 520, 1001, 1024, 2823, 4096, 4097, 4104, 8192, 8200, 11001, 16384, 16385, 16392, 20000, 32767, 32768,
          32769, 32776, 40000]


def depth(width):
    return 26 + max(16, -(-width // 1024))


def _case(n, w, kind, seed, mean=0.3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, w), generator=g) * torch.exp(torch.randn((n, 1), generator=g)) + mean * torch.randn((n, 1), generator=g)
    return x, torch.randn((n, w), generator=g), 1 + 0.3 * torch.randn((1, w), generator=g), torch.randn((1, w), generator=g)


def _forward_reference(x, w, b, eps):
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + eps)
    xh = (x - mean) * rstd
    return mean, rstd, xh * w + b


def _check_forward(x, w, b, eps, y, mean, rstd, kind):
    wm, wr, wy = _forward_reference(x, w, b, eps)
    d = depth(x.shape[1])
    size = x.abs().mean(1, keepdim=True)
    dmean = (d + 2) * U * size                                                  # sum and quotient
    assert_within(mean, wm[:, 0], dmean[:, 0] + 1e-300, "mean")
    # the squared deviations: relative d U and twice the two roundings of a deviation; the error of the mean enters squared
    # (deviations sum to zero, but for what the rounding of each leaves: 2 dmean U |deviations|, below the rest); half of it in rstd, and rsqrtf
    dvar = dmean ** 2 * wr ** 2
    drel = (d + 6) / 2 * U + dvar + 4 * U
    assert_within(rstd, wr[:, 0], (drel * wr)[:, 0], "rstd")
    xh = (x - wm) * wr
    tol = (drel + 4 * U) * (xh * w).abs() + 1.01 * dmean * wr * w.abs() + 2 * U * (wy.abs() + b.abs())
    assert_within(y, wy, tol + half_step(kind) * (wy.abs() + tol) + tiny(kind), "y")


def _check_backward(x, dy, w, mean, rstd, dx, dw, db, kind, rows_deep):
    n, width = x.shape
    xh, g = (x - mean[:, None]) * rstd[:, None], dy * w
    r, c1, c2 = rstd[:, None], g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    want = r * (g - c1 - xh * c2)
    d = depth(width)
    a1, a2 = g.abs().mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
    # g once rounded; xh twice; c1 by d + 2, c2 by d + 5 roundings; four more in the difference and its product
    tol = U * r * (6 * g.abs() + (d + 6) * a1 + (d + 12) * xh.abs() * a2)
    if dx is not None:
        assert_within(dx, want, tol + half_step(kind) * (want.abs() + tol) + tiny(kind), "dx")
    if dw is not None:
        assert_within(dw, (dy * xh).sum(0), (rows_deep + 4) * U * (dy * xh).abs().sum(0) + 1e-300, "dweight")
        assert_within(db, dy.sum(0), rows_deep * U * dy.abs().sum(0) + 1e-300, "dbias")


def _rows_deep(n):
    """roundings of a column's sum: the rows of a block one after the other (at least 148 blocks of at least one row each where there are
    so many, eight rows in turn in narrow ones), its planes by 32 threads and a tree"""
    return -(-n // 148) + 8 + 148 + 6


def _run(n, width, kind, ykind="", wkind="f32", pad=0, offset=0, packed=False, seed=None, affine=True, checkpoint=False):
    ykind = ykind or kind
    x, dy, w, b = _case(n, width, kind, seed if seed is not None else n * 7 + width)
    X, DY = Matrix(n, width, kind, pad, offset, x), Matrix(n, width, ykind, pad, offset, dy)
    W, B = Matrix(1, width, wkind, 0, offset, w), Matrix(1, width, wkind, 0, offset, b)
    Y, DX = Matrix(n, width, ykind, pad, offset), Matrix(n, width, kind, pad, offset)
    DW, DB = Matrix(1, width, "f32", 0, offset), Matrix(1, width, "f32", 0, offset)
    mean, rstd = (torch.full((n,), float("nan"), device="cuda") for _ in range(2))
    K = PackedMatrix(n, width, extra=pad % 2) if checkpoint or packed else None
    eps = 1e-5
    layernorm_forward(X.rows, n, width, Y.rows, W.rows if affine else None, B.rows if affine else None, eps, mean.data_ptr(), rstd.data_ptr(),
                      K.packed if K else None, stream=stream())
    wd, bd = (W.double(), B.double()) if affine else (torch.ones((1, width), dtype=torch.float64), torch.zeros((1, width), dtype=torch.float64))
    _check_forward(X.double(), wd, bd, eps, Y.double(), mean.double().cpu(), rstd.double().cpu(), ykind)
    Y.check_guards()
    source = X.double()
    if K:
        q, s = K.bytes()
        wq, ws = pack_reference(source.numpy())
        assert np.array_equal(s, ws) and same_codes(q, wq), "checkpoint"
        K.check_guards()
        if packed:
            source = torch.from_numpy(unpack_reference(q, s))
    ws, room = workspace(layernorm_workspace_bytes(n, width))
    layernorm_backward(DY.rows, None if packed else X.rows, K.packed if packed else None, n, width, mean.data_ptr(), rstd.data_ptr(), DX.rows,
                       W.rows if affine else None, DW.rows, DB.rows, stream=stream(), **room)
    _check_backward(source, DY.double(), wd, mean.double().cpu(), rstd.double().cpu(), DX.double(), DW.double()[0], DB.double()[0], kind, _rows_deep(n))
    for m in (DX, DW, DB):
        m.check_guards()
    return DX, DW, DB


@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_widths(width, kind):
    _run(5, width, kind, wkind=kind)


@pytest.mark.parametrize("n", [1, 2, 7, 9, 148, 149, 297, 1200, 2500])
@pytest.mark.parametrize("width", [96, 509, 1024, 4096])
def test_rows(n, width):
    _run(n, width, "bf16", wkind="f32")


@pytest.mark.parametrize("n,width", [(297, 4104), (703, 5000), (450, 6144), (299, 8192), (1000, 8200), (300, 12288), (301, 16376), (600, 16384)])
@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
def test_many_wide_rows(n, width, kind):
    _run(n, width, kind, wkind=kind, pad=8 * (n % 2), offset=16)


def test_many_wide_rows_of_other_types():
    _run(333, 8192, "bf16", ykind="f32", wkind="f32")
    _run(333, 6144, "f32", ykind="bf16", wkind="f16")
    _run(333, 5008, "bf16", affine=False)
    _run(333, 4800, "f32", packed=True)


def test_many_wide_rows_without_statistics_and_with_weights_off_every_boundary():
    n, width = 500, 7176
    x, _, w, b = _case(n, width, "bf16", 5)
    X, Y, W, B = Matrix(n, width, "bf16", values=x), Matrix(n, width, "bf16"), Matrix(1, width, "bf16", offset=1, values=w), Matrix(1, width, "bf16", offset=3, values=b)
    layernorm_forward(X.rows, n, width, Y.rows, W.rows, B.rows, 1e-5, stream=stream())
    got = Y.double()
    Y.check_guards()
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    layernorm_forward(X.rows, n, width, Y.rows, W.rows, B.rows, 1e-5, mean.data_ptr(), rstd.data_ptr(), stream=stream())
    assert torch.equal(got, Y.double())
    _check_forward(X.double(), W.double(), B.double(), 1e-5, got, mean.double().cpu(), rstd.double().cpu(), "bf16")


def test_many_wide_rows_with_infinities_stay_alone():
    n, width = 400, 8192
    x, _, w, b = _case(n, width, "bf16", 6)
    X, Y, W, B = Matrix(n, width, "bf16", values=x), Matrix(n, width, "bf16"), Matrix(1, width, "f32", values=w), Matrix(1, width, "f32", values=b)
    layernorm_forward(X.rows, n, width, Y.rows, W.rows, B.rows, 1e-5, stream=stream())
    want = Y.double()
    bad = torch.tensor([0, 7, 148, 399])
    X.t[bad.cuda(), torch.tensor([0, 8191, 4000, 1023]).cuda()] = torch.tensor([float("inf"), float("nan"), float("-inf"), float("nan")], dtype=torch.bfloat16, device="cuda")
    layernorm_forward(X.rows, n, width, Y.rows, W.rows, B.rows, 1e-5, stream=stream())
    got, rest = Y.double(), torch.ones(n, dtype=torch.bool)
    rest[bad] = False
    assert torch.equal(got[rest], want[rest]) and bool(torch.isnan(got[bad]).all())


def test_more_fp32_rows_than_the_second_level_cache_holds():
    _run(9501, 2536, "f32")


@pytest.mark.parametrize("kind,ykind,wkind", [("f32", "bf16", "f32"), ("bf16", "f32", "bf16"), ("f16", "bf16", "f16"), ("f32", "f16", "bf16")])
@pytest.mark.parametrize("width,pad,offset", [(1024, 0, 0), (1024, 8, 8), (1024, 3, 1), (401, 5, 3), (8200, 0, 0)])
def test_types_strides_offsets(kind, ykind, wkind, width, pad, offset):
    _run(13, width, kind, ykind, wkind, pad, offset)


@pytest.mark.parametrize("width", [8, 120, 128, 136, 512, 777, 1024, 4096, 5000, 8192, 8201, 16384, 17000, 17001, 33000, 33001])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_from_the_checkpoint(width, kind):
    _run(19, width, kind, packed=True, pad=0 if width % 16 else 8)


@pytest.mark.parametrize("width,pad", [(256, 1), (2048, 3)])
def test_checkpoint_of_unaligned_rows(width, pad):
    _run(6, width, "bf16", pad=pad, checkpoint=True)


def test_checkpoint_of_infinities_and_nans():
    """fp32 rows are packed in the norm's own pass: the same bytes as by pack8"""
    x, _, _, _ = _case(9, 1024, "f32", 2)
    x[1, 130], x[2, 0], x[3, 1000], x[4], x[5, 256:384] = float("inf"), float("nan"), -float("inf"), 0.0, float("nan")
    X, Y, K = Matrix(9, 1024, "f32", values=x), Matrix(9, 1024, "f32"), PackedMatrix(9, 1024)
    layernorm_forward(X.rows, 9, 1024, Y.rows, checkpoint=K.packed, stream=stream())
    q, s = K.bytes()
    wq, ws = pack_reference(x.double().numpy())
    assert np.array_equal(s, ws) and same_codes(q, wq)


def test_without_weights():
    _run(31, 640, "f32", affine=False)


@pytest.mark.parametrize("width", [100, 3000, 20000])
def test_only_what_is_wanted(width):
    n, kind = 11, "f32"
    x, dy, w, b = _case(n, width, kind, 5)
    X, DY, W = Matrix(n, width, kind, values=x), Matrix(n, width, kind, values=dy), Matrix(1, width, kind, values=w)
    mean, rstd = X.t.mean(1), torch.rsqrt(X.t.var(1, unbiased=False) + 1e-5)
    both = layernorm_workspace_bytes(n, width)
    for dx, dw, db in [(1, 0, 0), (0, 1, 0), (0, 0, 1), (0, 1, 1), (0, 0, 0)]:
        DX, DW, DB = Matrix(n, width, kind), Matrix(1, width, kind), Matrix(1, width, kind)
        ws, room = workspace(both) if dw or db else (None, {})
        layernorm_backward(DY.rows, X.rows, None, n, width, mean.data_ptr(), rstd.data_ptr(), DX.rows if dx else None, W.rows,
                           DW.rows if dw else None, DB.rows if db else None, stream=stream(), **room)
        torch.cuda.synchronize()
        d = X.double(), DY.double(), W.double(), mean.double().cpu(), rstd.double().cpu()
        xh = (d[0] - d[3][:, None]) * d[4][:, None]
        if dx:
            _check_backward(*d, DX.double(), None, None, kind, 0)
        if dw:
            assert_within(DW.double()[0], (d[1] * xh).sum(0), 200 * U * (d[1] * xh).abs().sum(0), "dweight")
        if db:
            assert_within(DB.double()[0], d[1].sum(0), 200 * U * d[1].abs().sum(0), "dbias")


def test_no_rows_gives_zero_sums():
    DW, DB, X = Matrix(1, 300, "f32"), Matrix(1, 300, "bf16"), Matrix(1, 300, "f32")
    ws, room = workspace(layernorm_workspace_bytes(0, 300))
    layernorm_backward(X.rows, X.rows, None, 0, 300, 0, 0, None, None, DW.rows, DB.rows, stream=stream(), **room)
    assert bool((DW.t == 0).all()) and bool((DB.t == 0).all())


def test_rows_with_infinities_and_nans_stay_alone():
    """a row with a NaN or an infinity is NaN, its neighbours in the same block are not; a constant row is the bias"""
    n, w = 40, 512
    x, _, wt, b = _case(n, w, "f32", 9)
    x[3, 17], x[20, 0], x[5] = float("nan"), float("inf"), 2.5
    X, Y, W, B = Matrix(n, w, "f32", values=x), Matrix(n, w, "f32"), Matrix(1, w, "f32", values=wt), Matrix(1, w, "f32", values=b)
    layernorm_forward(X.rows, n, w, Y.rows, W.rows, B.rows, stream=stream())
    y = Y.t.cpu()
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[20]).all())
    rest = [i for i in range(n) if i not in (3, 20)]
    assert bool(torch.isfinite(y[rest]).all()) and bool((y[5] == b[0]).all())


def test_large_mean_small_spread():
    """the variance comes from deviations, not from a difference of squares"""
    n, w = 6, 1000
    g = torch.Generator().manual_seed(1)
    x = 1000 + torch.randn((n, w), generator=g) * 0.01
    X, Y = Matrix(n, w, "f32", values=x), Matrix(n, w, "f32")
    mean, rstd = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    layernorm_forward(X.rows, n, w, Y.rows, eps=1e-12, mean_ptr=mean.data_ptr(), rstd_ptr=rstd.data_ptr(), stream=stream())
    one, zero = torch.ones((1, w), dtype=torch.float64), torch.zeros((1, w), dtype=torch.float64)
    _check_forward(X.double(), one, zero, 1e-12, Y.double(), mean.double().cpu(), rstd.double().cpu(), "f32")


def test_gradient_against_differences():
    """dx, dw, db of sum(dy y) against central differences of the forward formula in 64 bits"""
    n, w = 3, 24
    DX, DW, DB = _run(n, w, "f32", seed=3)
    x, dy, wt, b = (t.double() for t in _case(n, w, "f32", 3))
    loss = lambda x, wt, b: (dy * _forward_reference(x, wt, b, 1e-5)[2]).sum()
    h = 1e-5
    for t, got, k in ((x, DX, 0), (wt, DW, 1), (b, DB, 2)):
        for i in range(0, t.numel(), 5):
            args = [x.clone(), wt.clone(), b.clone()]
            args[k].view(-1)[i] += h
            up = loss(*args)
            args[k].view(-1)[i] -= 2 * h
            diff = (up - loss(*args)) / (2 * h)
            # central differences: h^2 times a third derivative of order 10, and roundings 1e-16 / h
            assert abs(float(got.t.reshape(-1)[i]) - float(diff)) <= 1e-4 * max(1.0, abs(float(diff)))


def test_same_bits_on_every_run():
    a = _run(700, 1024, "bf16", seed=1)
    b = _run(700, 1024, "bf16", seed=1)
    assert all(torch.equal(p.t, q.t) for p, q in zip(a, b))
