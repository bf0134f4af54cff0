"""Every width has a kernel, whatever the types and the alignment: gradients of three rows at all of 1 ... 16384 columns.

Three rows of small whole numbers with mean 0 and rstd 1: dw = sum dy x and db = sum dy are exact in fp32, and in bf16 as long as they are
below 2^8."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("dtype,wdtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
def test_every_width(dtype, wdtype, shift):
    g = torch.Generator().manual_seed(80)
    x, dy = (torch.randint(-4, 5, (3, 16392), generator=g).to(dtype).cuda() for _ in range(2))
    w = torch.randint(-2, 3, (16392,), generator=g).to(wdtype).cuda()
    dw_all, db_all = (dy.float() * x.float()).sum(0).to(wdtype), dy.float().sum(0).to(wdtype)
    mean, rstd = torch.zeros(3, device="cuda"), torch.ones(3, device="cuda")
    dx = torch.empty_like(x)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    wrong = torch.zeros((), dtype=torch.int64, device="cuda")
    for cols in range(1, 16385):
        at = slice(shift, shift + cols)
        a, b = dw[at], db[at]
        hb.layer_norm_backward(dy[:, at], x[:, at], w[at], mean, rstd, dx[:, at], a, b)
        wrong += (a != dw_all[at]).sum() + (b != db_all[at]).sum()
    assert int(wrong) == 0
    assert hb.layer_norm_status() == 0
