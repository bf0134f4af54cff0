"""A sequence's bits are its own: whatever finite values its neighbours hold, large scores among them.

Tiles have 128 rows; the last tile of a sequence also holds rows behind it, whose queries belong to the next sequence or to
nobody, and its scores with the keys of this one may be of any size."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from test_packed_gpu import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(4, 4), (8, 2), (3, 1)])
@pytest.mark.parametrize("lens", [(300, 200), (700, 1, 130), (205, 0, 333)])
def test_large_scores_of_the_rows_behind(lens, heads, kv_heads, dim, causal):
    q, k, v, cu = make(lens, heads, kv_heads, dim, 40, tail=140, fused=False)
    n = lens[0]
    # keys grow along the sequence, so that the rows behind it find ever larger scores in each block of keys
    k[:n] = (k[:n].float() * torch.linspace(0.2, 1.5, n, device="cuda")[:, None, None]).bfloat16()
    dout = torch.randn(q.shape, device="cuda").bfloat16()
    want = None
    for gain in (0.0, 1.0, 40.0):
        q2 = q.clone()
        q2[n:] *= gain
        out, lse = torch.zeros_like(q), torch.zeros((heads, q.shape[0]), device="cuda")
        hb.packed_forward(q2, k, v, out, cu, lse=lse, causal=causal)
        grads = [torch.zeros_like(t) for t in (q, k, v)]
        hb.packed_backward(dout, q2, k, v, out, lse, *grads, cu, causal=causal)
        got = [out[:n], lse[:, :n]] + [g[:n] for g in grads]
        want = want or got
        for name, a, b in zip(("out", "lse", "dq", "dk", "dv"), got, want):
            assert torch.equal(a, b), (name, gain, float((a.float() - b.float()).abs().max()))
    assert hb.packed_status() == 0
