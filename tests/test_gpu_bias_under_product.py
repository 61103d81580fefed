"""The gradient of a linear's bias is summed under the product of its weights' gradient: of the values that the kernel before the call wrote,
not of those that were there before, however the call is made; and its mark in the workspace is gone behind it."""
import pytest
import torch

import paper_1909_05840_b200 as qb
from test_gpu_interrupted_calls import run_first_launch

pytestmark = pytest.mark.gpu
# one launch for few columns and rows, rows of any length, more tiles than pairs of SMs, a product in parts
SIZES = [(613, 16, 768), (401, 9, 64), (4000, 1024, 1024), (3001, 2056, 520), (6144, 4096, 2048), (20000, 264, 264)]


def begun(ws):
    return int(ws[48:52].view(torch.int32).item())


def values(M, N, K):
    """Whole numbers, other ones for each i, whose sums are exact."""
    base = torch.randint(-3, 4, (M, N), device="cuda").bfloat16()
    x = torch.randint(-2, 3, (M, K), device="cuda").bfloat16()
    return [(base + i) for i in range(-4, 5)], x


@pytest.mark.parametrize("M,N,K", SIZES)
def test_other_values_at_the_same_address(M, N, K):
    ws = qb.linear_workspace(M, N, K)
    dys, x = values(M, N, K)
    want = [dy.double().sum(0).float() for dy in dys]
    weights = [(dy.float().t() @ x.float()) for dy in dys]
    buffer, kept = torch.empty_like(dys[0]), []
    for i in list(range(len(dys))) * 3:
        buffer.copy_(dys[i])
        kept.append((i, *qb.linear_grad_w(buffer, x, ws)))
        buffer.fill_(100.0)
    for i, dw, db in kept:
        assert torch.equal(db, want[i]) and torch.equal(dw, weights[i])
    assert begun(ws) == 0 and qb.read_status(ws) == qb.QB_OK


@pytest.mark.parametrize("M,N,K", SIZES[:3])
def test_two_graphs_over_one_workspace(M, N, K):
    """The write of the buffer is in the graph, so that nothing comes between it and the product; replays in turn."""
    ws = qb.linear_workspace(M, N, K)
    dys, x = values(M, N, K)
    want = [dy.double().sum(0).float() for dy in dys]
    source, buffer = torch.empty_like(dys[0]), torch.empty_like(dys[0])
    qb.linear_grad_w(dys[0], x, ws)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            buffer.copy_(source)
            _, db = qb.linear_grad_w(buffer, x, ws)
        graphs.append((graph, db))
    for i in list(range(len(dys))) * 2:
        source.copy_(dys[i])
        graph, db = graphs[i & 1]
        graph.replay()
        assert torch.equal(db, want[i])
        _, eager = qb.linear_grad_w(dys[-1 - i], x, ws)
        assert torch.equal(eager, want[-1 - i])
    assert begun(ws) == 0


def test_behind_a_call_that_was_cut_short():
    """The product of a call whose second launch never ran leaves its mark; the next calls do not take it for theirs."""
    M, N, K = SIZES[0]
    ws = qb.linear_workspace(M, N, K)
    dys, x = values(M, N, K)
    for _ in range(2):
        run_first_launch(lambda: qb.linear_grad_w(dys[0], x, ws))
        assert begun(ws) != 0
        for i, dy in enumerate(dys):
            assert torch.equal(qb.linear_grad_w(dy, x, ws)[1], dy.double().sum(0).float()), i
        assert begun(ws) == 0
