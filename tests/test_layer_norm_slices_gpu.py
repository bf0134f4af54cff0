"""Layer norm on tensors that lie side by side in one buffer: the same bits as apart, and nothing else touched."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("rows,cols,gap", [(1, 64, 0), (700, 64, 0), (700, 63, 1), (300, 777, 0), (300, 777, 3), (999, 1024, 8), (50, 5001, 0), (40, 10000, 0), (30, 9001, 5)])
def test_side_by_side(rows, cols, gap, dtype):
    g = torch.Generator().manual_seed(rows + cols)
    x, dy = (torch.randn((rows, cols), generator=g).to(dtype).cuda() for _ in range(2))
    w, b = (torch.randn((cols,), generator=g).cuda() for _ in range(2))
    if dtype == torch.bfloat16:
        w, b = w.bfloat16(), b.bfloat16()
    dw, db = torch.empty_like(w), torch.empty_like(w)
    mean, rstd = (torch.empty(rows, device="cuda") for _ in range(2))

    width = cols + gap
    wide = torch.full((rows, 4 * width), 7.0, dtype=dtype, device="cuda")
    x2, y2, dy2, dx2 = (wide[:, i * width:i * width + cols] for i in range(4))
    x2.copy_(x)
    dy2.copy_(dy)
    # the same alignment and path on both sides: tensors apart are slices of wide buffers of their own
    apart = [torch.full_like(wide, 7.0)[:, i * width:i * width + cols] for i in range(4)]
    apart[0].copy_(x)
    apart[2].copy_(dy)
    hb.layer_norm(apart[0], w, b, apart[1], mean, rstd)
    hb.layer_norm_backward(apart[2], apart[0], w, mean, rstd, apart[3], dw, db)
    for _ in range(3):
        dw2, db2 = torch.empty_like(w), torch.empty_like(w)
        hb.layer_norm(x2, w, b, y2)
        hb.layer_norm_backward(dy2, x2, w, mean, rstd, dx2, dw2, db2)
        for got, want in zip((x2, y2, dy2, dx2, dw2, db2), (x, apart[1], dy, apart[3], dw, db)):
            assert torch.equal(got, want)
        for i in range(4):
            assert (wide[:, i * width + cols:(i + 1) * width] == 7.0).all()
    assert hb.layer_norm_status() == 0
