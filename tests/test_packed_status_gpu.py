"""What packed_status promises: that the kernels before it, on whatever stream, are over when it answers."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from test_packed_gpu import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("backward", [False, True])
def test_status_waits_for_work_on_other_streams(backward):
    q, k, v, cu = make((8192, 4096, 8192), 16, 4, 128, 30)   # 60 calls take tens of milliseconds
    out, lse = torch.empty_like(q), torch.empty((16, q.shape[0]), device="cuda")
    hb.packed_forward(q, k, v, out, cu, lse=lse)
    grads = [torch.empty_like(t, memory_format=torch.contiguous_format) for t in (q, k, v)]
    dout = torch.randn(out.shape, device="cuda").bfloat16()
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    torch.cuda.synchronize()
    for _ in range(60):
        if backward:
            hb.packed_backward(dout, q, k, v, out, lse, *grads, cu, stream=side)
        else:
            hb.packed_forward(q, k, v, out, cu, lse=lse, stream=side)
    done.record(side)
    assert hb.packed_status() == 0
    assert done.query()
