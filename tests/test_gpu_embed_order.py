"""Tokens that the kernel directly before the gradient's call has written, uncaptured: its kernels start while their predecessors still run."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_1711_01348_b200 import Rows, embed_backward, embed_workspace_bytes  # noqa: E402
from tests.operator_util import Matrix, stream, workspace  # noqa: E402

NAN = float("nan")


@pytest.mark.parametrize("n", [1000, 30000])
@pytest.mark.parametrize("bits", [32, 64])
def test_tokens_written_directly_before_the_call(n, bits):
    """the rows to be cleared are found beside the sort: by the tokens that the kernel before has written, in a buffer that every call reads"""
    v, width, turns, kind = 20000, 32, 12, torch.int32 if bits == 32 else torch.int64
    g = torch.Generator().manual_seed(n)
    sources = [torch.randint(-1, v, (n,), generator=g).to(kind).cuda() for _ in range(turns)]
    DY = Matrix(n, width, "f32", values=torch.randint(-4, 5, (n, width), generator=g).float())
    tables = [torch.full((v, width), NAN, device="cuda") for _ in range(turns)]
    ws, room = workspace(embed_workspace_bytes(n, v, width))
    t = torch.zeros(n, dtype=kind, device="cuda")
    torch.cuda.synchronize()
    for source, table in zip(sources, tables):
        torch.add(source, 0, out=t)
        embed_backward(t.data_ptr(), bits, n, DY.rows, v, width, 1.0, Rows(table.data_ptr(), width, "f32"), stream=stream(), **room)
    for source, table in zip(sources, tables):
        live = source >= 0
        want = torch.zeros((v, width), device="cuda").index_add_(0, source[live].long(), DY.t[live])
        assert torch.equal(table, want)
