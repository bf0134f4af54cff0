"""Keys that a row does not see, or whose weight is nothing, leave no trace of their values, the largest finite ones among them."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from test_packed_gpu import make

pytestmark = pytest.mark.gpu
TOP = float(torch.finfo(torch.bfloat16).max)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (8, 2), (3, 1)])
@pytest.mark.parametrize("n,seen", [(300, 200), (128, 1), (77, 60), (700, 385), (129, 128)])
def test_causal_rows_do_not_feel_later_values(n, seen, heads, kv_heads, dim):
    q, k, v, cu = make((n,), heads, kv_heads, dim, 90, fused=False)
    want = None
    for later in (0.0, 1.0, TOP):
        v[seen:] = later
        out, lse = torch.zeros_like(q), torch.zeros((heads, n), device="cuda")
        hb.packed_forward(q, k, v, out, cu, lse=lse)
        got = out[:seen], lse[:, :seen]
        want = want or got
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert hb.packed_status() == 0


@pytest.mark.parametrize("dim", [64, 128])
def test_weights_far_below_the_smallest_number(dim):
    """Every key but the first scores 400 less (2^-577): the output is the first one's value, whatever the others'."""
    n = 256
    q, k, v = (torch.zeros((n, 1, dim), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    q[:, 0, 0] = 1.0
    k[1:, 0, 0] = -400.0
    v[0], v[1:] = 1.5, TOP
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    hb.packed_forward(q, k, v, out, cu, causal=False, scale=1.0)
    assert (out == 1.5).all()
