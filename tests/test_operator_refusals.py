"""What the operators refuse, before anything is launched; and what they accept up to the launch (no GPU here: the launch fails)."""
import ctypes as C

import pytest
import torch

from paper_1711_01348_b200 import (Packed, Rows, TadError, embed_backward, embed_forward, embed_workspace_bytes, layernorm_backward,
                                   layernorm_forward, layernorm_workspace_bytes, lib, matmul8, matmul8_workspace_bytes, pack8,
                                   repack8, unpack8)

P = 1 << 20          # a fake pointer, aligned to everything
ROOM = dict(workspace_ptr=P, workspace_bytes=1 << 40)

fake = pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers must not reach a GPU")


def _r(ptr=P, stride=100, kind="f32"):
    return Rows(ptr, stride, kind)


def _p(q=P, s=P, qs=112, ss=4):
    return Packed(q, s, qs, ss)


def _bad_type():
    r = _r()
    r.type = 3
    return r


def _reserved():
    r = _r()
    r.reserved = 1
    return r


BAD_ROWS = [_r(ptr=0), _r(stride=99), _r(ptr=P + 2), _r(ptr=P + 1, kind="bf16"), _bad_type(), _reserved(), None]
BAD_PACKED = [_p(q=0), _p(s=0), _p(qs=96), _p(qs=104), _p(q=P + 8), _p(s=P + 2), _p(ss=0), _p(ss=5), None]


def _refused(call, code="TAD_ERR_INVALID_ARG"):
    with pytest.raises(TadError) as e:
        call()
    assert e.value.code == code and str(e.value).split(": ", 1)[1]


@fake
@pytest.mark.parametrize("bad", BAD_ROWS)
def test_bad_matrices(bad):
    good = _r()
    _refused(lambda: pack8(bad, 3, 100, _p()))
    _refused(lambda: unpack8(_p(), 3, 100, bad))
    _refused(lambda: layernorm_forward(bad, 3, 100, good))
    _refused(lambda: layernorm_forward(good, 3, 100, bad))
    _refused(lambda: layernorm_backward(bad, good, None, 3, 100, P, P, good))
    _refused(lambda: embed_forward(P, 32, 3, bad, 7, 100, 1.0, good))
    _refused(lambda: embed_forward(P, 32, 3, good, 7, 100, 1.0, bad))
    _refused(lambda: embed_backward(P, 32, 3, bad, 7, 100, 1.0, good, **ROOM))
    _refused(lambda: embed_backward(P, 32, 3, good, 7, 100, 1.0, bad, **ROOM))
    _refused(lambda: matmul8(_p(), _p(), 5, 100, 100, bad, **ROOM))
    if bad is not None:
        _refused(lambda: layernorm_backward(good, bad, None, 3, 100, P, P, good))
        _refused(lambda: layernorm_backward(good, good, None, 3, 100, P, P, bad))


@fake
@pytest.mark.parametrize("bad", [b for b in BAD_ROWS if b is not None and b.stride == 100])
def test_bad_vectors(bad):
    good = _r()
    _refused(lambda: layernorm_forward(good, 3, 100, good, weight=bad))
    _refused(lambda: layernorm_forward(good, 3, 100, good, bias=bad))
    for name in ("weight", "dweight", "dbias"):
        _refused(lambda: layernorm_backward(good, good, None, 3, 100, P, P, good, **{name: bad}, **ROOM))


@fake
@pytest.mark.parametrize("bad", BAD_PACKED)
def test_bad_packed_matrices(bad):
    good = _r()
    _refused(lambda: pack8(good, 3, 100, bad))
    _refused(lambda: unpack8(bad, 3, 100, good))
    _refused(lambda: repack8(bad, 100, 100, _p()))
    _refused(lambda: repack8(_p(), 100, 100, bad))
    _refused(lambda: matmul8(bad, _p(), 100, 100, 100, good, **ROOM))
    _refused(lambda: matmul8(_p(), bad, 100, 100, 100, good, **ROOM))
    if bad is not None:
        _refused(lambda: layernorm_forward(good, 3, 100, good, checkpoint=bad))
        _refused(lambda: layernorm_backward(good, None, bad, 3, 100, P, P, good))


@fake
def test_arguments_of_their_own():
    r = _r()
    _refused(lambda: layernorm_forward(r, 3, 100, r, eps=-1.0))
    _refused(lambda: layernorm_forward(r, 3, 100, r, eps=float("nan")))
    _refused(lambda: layernorm_backward(r, r, _p(), 3, 100, P, P, r))          # both sources
    _refused(lambda: layernorm_backward(r, None, None, 3, 100, P, P, r))       # none
    _refused(lambda: layernorm_backward(r, r, None, 3, 100, 0, P, r))
    _refused(lambda: layernorm_backward(r, r, None, 3, 100, P, 0, r))
    _refused(lambda: layernorm_backward(r, r, None, 3, 100, P + 2, P, r))
    _refused(lambda: layernorm_backward(r, r, None, 3, 100, P, P + 1, r))
    _refused(lambda: layernorm_forward(r, 3, 100, r, mean_ptr=P + 2))
    _refused(lambda: layernorm_forward(r, 3, 100, r, rstd_ptr=P + 2))
    _refused(lambda: embed_forward(P, 16, 3, r, 7, 100, 1.0, r))
    _refused(lambda: embed_forward(0, 32, 3, r, 7, 100, 1.0, r))
    _refused(lambda: embed_forward(P + 4, 64, 3, r, 7, 100, 1.0, r))
    _refused(lambda: embed_forward(P, 32, 3, r, -1, 100, 1.0, r))
    for call in (lambda n, w: pack8(r, n, w, _p()), lambda n, w: unpack8(_p(), n, w, r), lambda n, w: layernorm_forward(r, n, w, r),
                 lambda n, w: embed_forward(P, 32, n, r, 7, w, 1.0, r), lambda n, w: matmul8(_p(), _p(), n, 100, w, r, **ROOM)):
        _refused(lambda: call(-1, 100))
        _refused(lambda: call(3, -1))
    big = Rows(P, 1 << 40, "f32")
    _refused(lambda: pack8(big, 1 << 31, 100, _p()), "TAD_ERR_UNSUPPORTED")
    _refused(lambda: layernorm_forward(big, 3, 1 << 24, big), "TAD_ERR_UNSUPPORTED")
    _refused(lambda: embed_forward(P, 32, 3, big, 1 << 31, 100, 1.0, big), "TAD_ERR_UNSUPPORTED")
    far = Packed(P, P, 1 << 30, 1 << 20)
    _refused(lambda: repack8(far, 1 << 24, 100, far), "TAD_ERR_UNSUPPORTED")
    # more blocks than a launch has: sizes beyond any memory, and the accesses with them
    _refused(lambda: pack8(big, (1 << 31) - 1, (1 << 24) - 1, far), "TAD_ERR_UNSUPPORTED")
    _refused(lambda: unpack8(far, (1 << 31) - 1, (1 << 24) - 1, big), "TAD_ERR_UNSUPPORTED")
    _refused(lambda: pack8(Rows(P + 4, 1 << 40, "f32"), (1 << 31) - 1, (1 << 24) - 1, far), "TAD_ERR_UNSUPPORTED")
    _refused(lambda: matmul8(far, far, (1 << 31) - 1, 1 << 20, 100, big, **ROOM), "TAD_ERR_UNSUPPORTED")


@fake
def test_workspaces():
    r = _r()
    for n in (1, 50, 5000):
        need = layernorm_workspace_bytes(n, 100)
        assert need > 0 and need % 256 == 0
        for room in ({}, dict(workspace_ptr=P, workspace_bytes=need - 1), dict(workspace_ptr=P + 128, workspace_bytes=1 << 30)):
            _refused(lambda: layernorm_backward(r, r, None, n, 100, P, P, r, dweight=r, **room), "TAD_ERR_WORKSPACE")
            _refused(lambda: embed_backward(P, 32, n, r, 7, 100, 1.0, r, **room), "TAD_ERR_WORKSPACE") if embed_workspace_bytes(n, 7, 100) >= need or not room else None
    need = matmul8_workspace_bytes(200, 100, 9000)
    assert need > 0
    wide = _p(qs=9008, ss=72)
    _refused(lambda: matmul8(wide, wide, 200, 100, 9000, r), "TAD_ERR_WORKSPACE")
    _refused(lambda: matmul8(wide, wide, 200, 100, 9000, r, workspace_ptr=P, workspace_bytes=need - 1), "TAD_ERR_WORKSPACE")
    assert layernorm_workspace_bytes(0, 10) == layernorm_workspace_bytes(10, 0) == embed_workspace_bytes(0, 5, 5) == matmul8_workspace_bytes(0, 5, 5) == 0
    assert layernorm_workspace_bytes(-1, 10) == embed_workspace_bytes(1 << 31, 5, 5) == matmul8_workspace_bytes(5, 5, 1 << 24) == 0


def test_nothing_to_do_is_no_launch():
    """sizes of zero need no data and no device"""
    none, p = Rows(0, 0, "bf16"), Packed(0, 0, 0, 0)
    pack8(none, 0, 0, p)
    unpack8(p, 0, 0, none)
    repack8(p, 0, 0, p)
    layernorm_forward(none, 0, 0, none)
    layernorm_backward(none, none, None, 0, 0, 0, 0, none)
    embed_forward(0, 32, 0, none, 0, 0, 1.0, none)
    embed_backward(0, 64, 0, none, 0, 0, 1.0, none)
    embed_backward(0, 64, 0, none, 5, 0, 1.0, none, accumulate=True)
    matmul8(p, p, 0, 0, 0, none)
    with pytest.raises(TadError):
        layernorm_forward(none, 0, 0, none, eps=-1.0)


@fake
def test_good_calls_reach_the_launch():
    r = _r()
    for call in (lambda: pack8(r, 3, 100, _p()), lambda: unpack8(_p(), 3, 100, r), lambda: repack8(_p(), 100, 100, _p()),
                 lambda: layernorm_forward(r, 3, 100, r, r, r, checkpoint=_p()), lambda: layernorm_backward(r, r, None, 3, 100, P, P, r),
                 lambda: layernorm_backward(r, None, _p(), 3, 100, P, P, r, r, r, r, **ROOM), lambda: embed_forward(P, 64, 3, r, 7, 100, 1.0, r),
                 lambda: embed_backward(P, 32, 3, r, 7, 100, 1.0, r, **ROOM), lambda: matmul8(_p(), _p(), 2, 100, 100, r),
                 lambda: matmul8(_p(), _p(), 100, 100, 100, r, **ROOM)):
        _refused(call, "TAD_ERR_CUDA")


@fake
def test_lookups_beyond_a_launch():
    for offset in (0, 4):
        m = Rows(P + offset, 1 << 40, "f32")
        _refused(lambda: embed_forward(P, 32, (1 << 31) - 1, m, 7, (1 << 24) - 8, 1.0, m), "TAD_ERR_UNSUPPORTED")


def test_descriptors_have_the_layout_of_the_header():
    assert C.sizeof(Rows) == 24 and Rows.stride.offset == 8 and Rows.type.offset == 16
    assert C.sizeof(Packed) == 32 and Packed.q_stride.offset == 16 and Packed.scale_stride.offset == 24
    assert lib.tad_pack8.argtypes
