"""Helpers for the tests of the operators: matrices with strides, offsets and guards, packed matrices, and the definition of the
8-bit blocks in 64 bits (by search among all values of the format)."""
from __future__ import annotations

import numpy as np
import torch

from paper_1711_01348_b200 import Packed, Rows

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24                      # half a step of fp32, relative to the value
GUARD = 0.4375                      # what lies between rows and behind them (a value of all types)


def half_step(kind):
    return torch.finfo(TYPES[kind]).eps / 2


def tiny(kind):
    """half the smallest step of the type: what a rounding is off by at most where numbers are subnormal"""
    f = torch.finfo(TYPES[kind])
    return f.tiny * f.eps / 2


class Matrix:
    """n x width elements on the GPU, `pad` elements behind each row, the first `offset` elements into the buffer."""

    def __init__(self, n, width, kind, pad=0, offset=0, values=None):
        self.n, self.width, self.kind, self.stride, self.offset = n, width, kind, width + pad, offset
        self.buf = torch.full((offset + n * self.stride + 16,), GUARD, dtype=TYPES[kind], device="cuda")
        self.t = self.buf[offset:offset + n * self.stride].view(n, self.stride)[:, :width]
        if values is not None:
            self.t.copy_(values)
        self.rows = Rows(self.buf.data_ptr() + offset * self.buf.element_size(), self.stride, kind)

    def double(self):
        return self.t.double().cpu()

    def check_guards(self):
        b = self.buf.clone()
        b[self.offset:self.offset + self.n * self.stride].view(self.n, self.stride)[:, :self.width] = GUARD
        assert bool((b == GUARD).all()), "written outside the matrix"


class PackedMatrix:
    def __init__(self, n, width, extra=0, fill=0x55):
        self.n, self.width, self.nb = n, width, -(-width // 128)
        self.qs, self.ss = -(-max(width, 1) // 16) * 16 + 16 * extra, -(-max(self.nb, 1) // 4) * 4 + 4 * extra
        self.q = torch.full((max(n, 1), self.qs), fill, dtype=torch.uint8, device="cuda")
        self.s = torch.full((max(n, 1), self.ss), fill, dtype=torch.uint8, device="cuda")
        self.fill = fill
        self.packed = Packed(self.q.data_ptr(), self.s.data_ptr(), self.qs, self.ss)

    def put(self, q, s):
        self.q[:, :self.width] = torch.from_numpy(q).cuda()
        self.s[:, :self.nb] = torch.from_numpy(s).cuda()
        return self

    def bytes(self):
        return self.q[:self.n, :self.width].cpu().numpy(), self.s[:self.n, :self.nb].cpu().numpy()

    def check_guards(self):
        assert bool((self.q[:, self.width:] == self.fill).all()) and bool((self.s[:, self.nb:] == self.fill).all()), "written outside the matrix"


def e4m3_table():
    """values of the codes 0 .. 126 (127 is NaN), from the definition"""
    c = np.arange(127)
    e, f = c >> 3, c & 7
    return np.where(e > 0, (1 + f / 8.0) * 2.0 ** (e - 7.0), f / 8.0 * 2.0 ** -6)


TABLE = e4m3_table()


def pack_reference(x):
    """(codes, exponent bytes) of a float64 matrix; NaN codes are 0x7f"""
    x = np.asarray(x, dtype=np.float64)
    n, w = x.shape
    nb = -(-w // 128)
    q, s = np.zeros((n, w), np.uint8), np.zeros((n, nb), np.uint8)
    mid = (TABLE[1:] + TABLE[:-1]) / 2
    for b in range(nb):
        part = x[:, b * 128:(b + 1) * 128]
        a = np.where(np.isfinite(part), np.abs(part), 0.0).max(axis=1)
        k = np.full(n, -126)
        for _ in range(300):                       # the least k >= -126 with a <= 448 2^k
            k = np.where(a > 448.0 * 2.0 ** k.astype(np.float64), k + 1, k)
        k = np.where(a == 0, 0, k)
        v = part / (2.0 ** k.astype(np.float64))[:, None]
        m = np.abs(v)
        code = np.searchsorted(mid, m, side="left")                    # ties: the lower neighbour ...
        tie = (code < 126) & np.isin(m, mid)
        code = np.where(tie & (code % 2 == 1), code + 1, code)         # ... unless the upper one is even
        code = code | np.where(np.signbit(v), 128, 0)
        q[:, b * 128:(b + 1) * 128] = np.where(np.isfinite(part), code, 0x7f)
        s[:, b] = k + 127
    return q, s


def unpack_reference(q, s):
    full = np.concatenate([TABLE, [np.nan]])
    v = full[q & 0x7f] * np.where(q & 0x80, -1.0, 1.0)
    e = np.repeat(s.astype(np.float64), 128, axis=1)[:, :q.shape[1]]
    return v * np.where(e == 255, np.nan, 2.0 ** (e - 127.0))


def same_codes(got, want):
    """codes are equal; a NaN is a NaN whatever its sign"""
    nan = (want & 0x7f) == 0x7f
    return np.array_equal((got & 0x7f) == 0x7f, nan) and np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want))


def stream():
    return torch.cuda.current_stream().cuda_stream


def workspace(n):
    """device memory full of NaNs, and its arguments"""
    t = torch.full((max(256, n),), 255, dtype=torch.uint8, device="cuda")
    return t, dict(workspace_ptr=t.data_ptr(), workspace_bytes=n)


def assert_within(got, want, tol, what):
    bad = ~((got - want).abs() <= tol)
    if bool(bad.any()):
        i = int(torch.argmax(torch.where(bad, (got - want).abs() / tol.clamp(min=1e-300), torch.zeros_like(tol))))
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} off; worst {got.flatten()[i]!r} for {want.flatten()[i]!r}, tolerance {tol.flatten()[i]!r}")
