"""A training step through all operators and a compiled expression: tokens are looked up, normalised (the norm's input is kept in 8 bits),
multiplied by packed weights, the rest of the layer is an expression; back through the expression's gradient, the two products of
the layer, the norm from its checkpoint and the lookup.  Every stage against its formula in 64 bits at the inputs that the stage before
has given it; then the whole step again on a stream of its own, and captured into a graph and replayed on new data: the same bits."""
import torch
import pytest

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import (Packed, Plan, Rows, embed_backward, embed_forward, embed_workspace_bytes, layernorm_backward,  # noqa: E402
                                   layernorm_forward, layernorm_workspace_bytes, matmul8, matmul8_workspace_bytes, pack8, repack8, unpack8)
from tests.operator_util import U, assert_within, half_step, pack_reference, same_codes, tiny, unpack_reference  # noqa: E402
from workloads.expr import Builder, unit  # noqa: E402

T, V, D, N = 300, 1000, 384, 520          # tokens, table, width, columns of the layer
FACTOR, EPS = 4.0, 1e-5


def _rows(t):
    return Rows(t.data_ptr(), t.stride(0), {torch.float32: "f32", torch.bfloat16: "bf16"}[t.dtype])


class _Eight:
    def __init__(self, n, w):
        self.w = w
        self.q = torch.zeros((n, -(-w // 16) * 16), dtype=torch.uint8, device="cuda")
        self.s = torch.full((n, -(-(-(-w // 128)) // 4) * 4), 127, dtype=torch.uint8, device="cuda")
        self.p = Packed(self.q.data_ptr(), self.s.data_ptr(), self.q.stride(0), self.s.stride(0))

    def bytes(self):
        return self.q[:, :self.w].cpu().numpy(), self.s[:, :-(-self.w // 128)].cpu().numpy()

    def values(self):
        return torch.from_numpy(unpack_reference(*self.bytes()))


def _expression():
    """f_tn = tanh(h_tn) v_n"""
    b = Builder("layer_end", [T, N], 0, ["h", "v"], [[T, N], [N]])
    b.bin("mul", b.un("tanh", b.load("h", [unit(2, (0, 1)), unit(2, (1, 1))])), b.load("v", [unit(2, (1, 1))]))
    return b.done()


class Step:
    def __init__(self, seed):
        d = dict(device="cuda")
        f32, bf16 = dict(dtype=torch.float32, **d), dict(dtype=torch.bfloat16, **d)
        self.tokens = torch.empty(T, dtype=torch.int64, **d)
        self.table, self.w, self.b = torch.empty((V, D), **bf16), torch.empty((1, D), **f32), torch.empty((1, D), **f32)
        self.weight, self.v, self.df = torch.empty((N, D), **f32), torch.empty(N, **f32), torch.empty((T, N), **f32)
        self.load(seed)
        self.x, self.y = torch.empty((T, D), **bf16), torch.empty((T, D), **bf16)
        self.mean, self.rstd = torch.empty(T, **f32), torch.empty(T, **f32)
        self.kept, self.y8, self.yt8 = _Eight(T, D), _Eight(T, D), _Eight(D, T)
        self.w8, self.wt8 = _Eight(N, D), _Eight(D, N)
        self.h, self.f = torch.empty((T, N), **f32), torch.empty((T, N), **f32)
        self.dh, self.dv = torch.empty((T, N), **f32), torch.empty(N, **f32)
        self.dh8, self.dht8 = _Eight(T, N), _Eight(N, T)
        self.dy, self.dweight = torch.empty((T, D), **bf16), torch.empty((N, D), **f32)
        self.dx, self.dw, self.db = torch.empty((T, D), **bf16), torch.empty((1, D), **f32), torch.empty((1, D), **f32)
        self.dtable, self.back = torch.empty((V, D), **f32), torch.empty((T, D), **bf16)
        self.plan = Plan(_expression())
        need = max(self.plan.workspace_bytes(), layernorm_workspace_bytes(T, D), embed_workspace_bytes(T, V, D), matmul8_workspace_bytes(T, N, D),
                   matmul8_workspace_bytes(T, D, N), matmul8_workspace_bytes(N, D, T), 256)
        self.ws = torch.full((need,), 255, dtype=torch.uint8, **d)

    def load(self, seed):
        g = torch.Generator().manual_seed(seed)
        r = lambda *s, scale=1.0: torch.randn(s, generator=g) * scale
        self.tokens.copy_(torch.randint(-2, V, (T,), generator=g))
        self.table.copy_(r(V, D))
        self.w.copy_(1 + r(1, D, scale=0.1))
        self.b.copy_(r(1, D, scale=0.1))
        self.weight.copy_(r(N, D, scale=D ** -0.5))
        self.v.copy_(r(N))
        self.df.copy_(r(T, N))

    def run(self):
        st, room = torch.cuda.current_stream().cuda_stream, dict(workspace_ptr=self.ws.data_ptr(), workspace_bytes=self.ws.numel())
        embed_forward(self.tokens.data_ptr(), 64, T, _rows(self.table), V, D, FACTOR, _rows(self.x), stream=st)
        layernorm_forward(_rows(self.x), T, D, _rows(self.y), _rows(self.w), _rows(self.b), EPS, self.mean.data_ptr(), self.rstd.data_ptr(), self.kept.p, stream=st)
        pack8(_rows(self.weight), N, D, self.w8.p, stream=st)
        pack8(_rows(self.y), T, D, self.y8.p, stream=st)
        matmul8(self.y8.p, self.w8.p, T, N, D, _rows(self.h), stream=st, **room)
        args = [self.h.data_ptr(), self.v.data_ptr()]
        self.plan.forward(args, self.f.data_ptr(), st, **room)
        self.plan.backward(args, self.df.data_ptr(), [self.dh.data_ptr(), self.dv.data_ptr()], stream=st, **room)
        pack8(_rows(self.dh), T, N, self.dh8.p, stream=st)
        repack8(self.dh8.p, T, N, self.dht8.p, stream=st)
        repack8(self.y8.p, T, D, self.yt8.p, stream=st)
        repack8(self.w8.p, N, D, self.wt8.p, stream=st)
        matmul8(self.dh8.p, self.wt8.p, T, D, N, _rows(self.dy), stream=st, **room)
        matmul8(self.dht8.p, self.yt8.p, N, D, T, _rows(self.dweight), stream=st, **room)
        layernorm_backward(_rows(self.dy), None, self.kept.p, T, D, self.mean.data_ptr(), self.rstd.data_ptr(), _rows(self.dx), _rows(self.w),
                           _rows(self.dw), _rows(self.db), stream=st, **room)
        embed_backward(self.tokens.data_ptr(), 64, T, _rows(self.dx), V, D, FACTOR, _rows(self.dtable), stream=st, **room)
        unpack8(self.kept.p, T, D, _rows(self.back), stream=st)

    OUT = ["x", "y", "mean", "rstd", "h", "f", "dh", "dv", "dy", "dweight", "dx", "dw", "db", "dtable", "back"]
    EIGHT = ["kept", "y8", "yt8", "w8", "wt8", "dh8", "dht8"]

    def outputs(self):
        torch.cuda.synchronize()
        return [getattr(self, n).clone() for n in self.OUT] + [x for n in self.EIGHT for x in (getattr(self, n).q.clone(), getattr(self, n).s.clone())]

    def clear(self):
        for n in self.OUT:
            getattr(self, n).fill_(float("nan"))


def _d(t):
    return t.double().cpu()


def _product_tolerance(a, b, k, kind, want):
    size = a.abs() @ b.abs().T
    tol = (-(-k // 32) * 66 + 20) * U * size                  # (as in the test of the product)
    return tol + half_step(kind) * (want.abs() + tol) + tiny(kind)


def test_every_stage():
    s = Step(1)
    s.run()
    torch.cuda.synchronize()
    tok, live = s.tokens.cpu(), (s.tokens.cpu() >= 0)
    x = torch.where(live[:, None], _d(s.table)[tok.clamp(0)] * FACTOR, torch.zeros((), dtype=torch.float64))
    assert torch.equal(_d(s.x), x)                             # (a power of two: exact)
    mean = x.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((x - mean) ** 2).mean(1, keepdim=True) + EPS)
    y = (x - mean) * rstd * _d(s.w) + _d(s.b)
    # fp32 statistics of 384 elements: 60 roundings of the largest partial results at most, far below those of bf16
    assert_within(_d(s.y), y, half_step("bf16") * y.abs() + 100 * U * (1 + y.abs()) * (1 + rstd * x.abs().mean(1, keepdim=True)), "y")
    for eight, source in ((s.kept, s.x), (s.y8, s.y), (s.w8, s.weight), (s.dh8, s.dh)):
        q, sc = pack_reference(_d(source).numpy())
        assert same_codes(eight.bytes()[0], q) and (eight.bytes()[1] == sc).all()
    for turned, eight in ((s.yt8, s.y8), (s.wt8, s.w8), (s.dht8, s.dh8)):
        q, sc = pack_reference(eight.values().numpy().T)
        assert same_codes(turned.bytes()[0], q) and (turned.bytes()[1] == sc).all()
    assert torch.equal(_d(s.back), s.kept.values())
    for out, a, b, kind in ((s.h, s.y8, s.w8, "f32"), (s.dy, s.dh8, s.wt8, "bf16"), (s.dweight, s.dht8, s.yt8, "f32")):
        want = a.values() @ b.values().T
        assert_within(_d(out), want, _product_tolerance(a.values(), b.values(), a.w, kind, want), "product")
    h, v, df = _d(s.h), _d(s.v), _d(s.df)
    for got, want, size in ((s.f, torch.tanh(h) * v, v.abs()), (s.dh, df * v / torch.cosh(h) ** 2, (df * v).abs()), (s.dv, (df * torch.tanh(h)).sum(0), (df * torch.tanh(h)).abs().sum(0))):
        assert_within(_d(got), want, 1e-4 * size + 1e-6, "expression")                     # (the library's stated tolerance of expressions)
    xk, m, r, dy, w = s.kept.values(), _d(s.mean)[:, None], _d(s.rstd)[:, None], _d(s.dy), _d(s.w)
    xh, g = (xk - m) * r, dy * w
    dx = r * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    size = r * (g.abs() + g.abs().mean(1, keepdim=True) + xh.abs() * (g * xh).abs().mean(1, keepdim=True))
    assert_within(_d(s.dx), dx, half_step("bf16") * dx.abs() + 60 * U * size + tiny("bf16"), "dx")
    assert_within(_d(s.dw)[0], (dy * xh).sum(0), 400 * U * (dy * xh).abs().sum(0), "dw")
    assert_within(_d(s.db)[0], dy.sum(0), 400 * U * dy.abs().sum(0), "db")
    at, dxd = tok[live], _d(s.dx)[live]
    want = torch.zeros((V, D), dtype=torch.float64).index_add_(0, at, dxd) * FACTOR
    size = torch.zeros((V, D), dtype=torch.float64).index_add_(0, at, dxd.abs()) * FACTOR
    assert_within(_d(s.dtable), want, 20 * U * size, "dtable")


def test_on_another_stream_and_captured():
    s = Step(2)
    s.run()
    first = s.outputs()
    s.clear()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        s.run()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, s.outputs()))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run()
    for seed in (3, 2):
        s.load(seed)
        s.clear()
        graph.replay()
        got = s.outputs()
        s.clear()
        s.run()
        assert all(torch.equal(a, b) for a, b in zip(got, s.outputs()))
    assert all(torch.equal(a, b) for a, b in zip(first, got))


def test_two_streams_with_workspaces_of_their_own():
    """calls on two streams at a time, each with its own buffers, give what they give alone"""
    a, b = Step(4), Step(5)
    want = []
    for s in (a, b):
        s.run()
        want.append(s.outputs())
        s.clear()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        for s, st in zip((a, b), streams):
            with torch.cuda.stream(st):
                s.run()
    torch.cuda.synchronize()
    for s, w in zip((a, b), want):
        assert all(torch.equal(x, y) for x, y in zip(w, s.outputs()))
