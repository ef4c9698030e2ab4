"""Workspaces of PositionBias.backward over rising lengths, with captured graphs that go on using smaller ones."""
import pytest

pytestmark = pytest.mark.gpu


def _grad(seed, n, heads=4, batch=2):
    import torch
    return torch.randint(-4, 5, (batch, heads, n, n), generator=torch.Generator().manual_seed(seed)).float().cuda()


def test_rising_lengths_hold_what_the_longest_needs():
    import torch
    import paper_2206_10581_amd as tt
    bias = tt.PositionBias(torch.zeros((32, 16), device="cuda"), tt.PositionBias.log_buckets(32, 2048).cuda())
    grad, out = torch.zeros((8, 16, 700, 700), device="cuda"), torch.empty((32, 16), device="cuda")

    def asked():                                               # what blocks hold beyond that is the allocator's own rounding
        return torch.cuda.memory_stats()["requested_bytes.all.current"]

    before = asked()
    for n in range(16, 700, 4):
        bias.backward(grad[:, :, :n, :n], out=out)
    assert asked() - before <= bias.workspace_bytes + 4096
    fixed = tt.PositionBias(bias.weight, bias.bucket_of)
    fixed.backward(grad, out=out)
    assert bias.workspace_bytes <= 1.5 * fixed.workspace_bytes


@pytest.mark.parametrize("grown", [False, True])
def test_graphs_keep_the_workspace_that_they_used(grown):
    """grown: the capture's own call is the first of its size.  Sums of whole numbers, which are exact."""
    import torch
    import paper_2206_10581_amd as tt
    of = tt.PositionBias.log_buckets(16, 64).cuda()
    bias, eager = (tt.PositionBias(torch.zeros((16, 4), device="cuda"), of) for _ in range(2))
    sizes, graphs = (40, 130, 300), []
    for n in sizes:
        grad, out = _grad(n, n), torch.zeros((16, 4), device="cuda")
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            bias.backward(grad[:, :, :9, :9] if grown else grad)
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            bias.backward(grad, out=out)
        graphs.append((graph, grad, out))
    bias.backward(_grad(1, 900))
    for k in range(4):
        other = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]   # what was given back is used again
        for graph, grad, out in graphs:
            grad.copy_(_grad(k, grad.shape[2]))
            graph.replay()
            want = eager.backward(grad, out=torch.empty_like(out))
            bias.backward(_grad(k, 20))
            torch.cuda.synchronize()
            assert torch.equal(out, want)
        assert all(bool(t.isnan().all()) for t in other)
