"""Packed attention's gradients where key tiles are few: a key tile's heads are then taken in parts, whose sums are added up
afterwards.  Inputs, reference and tolerances as for the whole groups."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from test_packed_backward_gpu import _check, _tensors
from test_packed_gpu import CANARY, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim,lens", [
    (8, 1, 128, (1000,)), (8, 1, 64, (129,)), (6, 1, 64, (200, 333)), (14, 2, 128, (640, 129, 1)), (32, 8, 64, (2048,)),
    (48, 8, 64, (92, 33, 90)),      # parts of one head
    (48, 8, 128, (700, 452)),       # parts of three
    (17, 1, 64, (30,) * 40),        # a group that only its heads divide
    (17, 1, 64, (30,) * 60),        # ... and more units than that is done for
    (64, 1, 64, (3, 0, 400, 128)),
])
def test_parts(heads, kv_heads, dim, lens, causal):
    _check(*make(lens, heads, kv_heads, dim, 9, lead=3, tail=5), causal)


@pytest.mark.parametrize("causal", [True, False])
def test_layouts_and_scale(causal):
    q, k, v, cu = make((300, 77), 8, 2, 64, 4)
    packed = torch.full((377, 12, 64), CANARY, dtype=torch.bfloat16, device="cuda")
    _check(q, k, v, cu, causal, scale=0.3, grads=[packed[:, :8], packed[:, 8:10], packed[:, 10:]])


@pytest.mark.parametrize("lead,tail", [(0, 0), (130, 300)])
def test_same_bits_again_whatever_the_workspace_held(lead, tail):
    q, k, v, cu = make((555, 130), 12, 2, 128, 6, lead=lead, tail=tail)
    dout, out, lse = _tensors(q, k, v, cu, True, 7)
    runs = []
    for fill in (0, 255):   # 255: every float a NaN
        ws = torch.full((hb.packed_workspace(q.shape[0], 12),), fill, dtype=torch.uint8, device="cuda")
        grads = [torch.full(t.shape, CANARY, dtype=torch.bfloat16, device="cuda") for t in (q, k, v)]
        graph = torch.cuda.CUDAGraph()
        hb.packed_backward(dout, q, k, v, out, lse, *grads, cu, workspace=ws)
        runs.append([g.clone() for g in grads])
        ws.fill_(fill)
        with torch.cuda.graph(graph):
            hb.packed_backward(dout, q, k, v, out, lse, *grads, cu, workspace=ws, stream=torch.cuda.current_stream())
        for g in grads:
            g.fill_(CANARY)
        graph.replay()
        torch.cuda.synchronize()
        runs.append(grads)
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))
    assert all((g[:lead] == CANARY).all() and (g[len(g) - tail:] == CANARY).all() for g in runs[0])
    assert hb.packed_status() == 0


@pytest.mark.parametrize("total,heads", [(129, 8), (4096, 8), (18000, 17), (18900, 2), (300, 1), (7, 4)])
def test_workspace_is_bounded(total, heads):
    n = hb.packed_workspace(total, heads)
    assert 8 * total * heads <= n <= 8 * total * heads + 256 + 160 * 2 ** 20
