"""Calls of the packed gradients that share a workspace, one right behind the other: each reads the statistics of its own."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from test_packed_gpu import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim,lens", [(4, 4, 128, (300,)), (8, 2, 64, (130, 77)), (3, 1, 128, (40, 260)), (16, 1, 64, (1000,))])
def test_one_workspace_for_calls_with_other_statistics(heads, kv_heads, dim, lens, causal):
    calls = []
    for seed in range(4):
        q, k, v, cu = make(lens, heads, kv_heads, dim, 70 + seed, gain=1.0 + seed)
        dout = torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)).bfloat16().cuda() * (seed + 1)
        out, lse = torch.empty_like(q), torch.empty((heads, q.shape[0]), device="cuda")
        hb.packed_forward(q, k, v, out, cu, lse=lse, causal=causal)
        want = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in (q, k, v)]
        hb.packed_backward(dout, q, k, v, out, lse, *want, cu, causal=causal)
        torch.cuda.synchronize()
        calls.append(((dout, q, k, v, out, lse), want, [torch.empty_like(t) for t in want], cu))
    shared = torch.empty(hb.packed_workspace(sum(lens), heads), dtype=torch.uint8, device="cuda")

    def run():
        for args, _, got, cu in calls:
            hb.packed_backward(*args, *got, cu, causal=causal, workspace=shared)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        run()
    for again in (run, graph.replay):
        for _ in range(20):
            for _, _, got, _ in calls:
                for t in got:
                    t.fill_(7.0)
            torch.cuda.synchronize()
            again()
            torch.cuda.synchronize()
            for _, want, got, _ in calls:
                assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert hb.packed_status() == 0
