"""The layer norm's bounded waits: one that runs out is reported once, and the device stays usable.  No kernel faults or hangs."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu


def _gradients():
    x, dy = (torch.randn((3000, 1024), device="cuda").bfloat16() for _ in range(2))
    w = torch.ones(1024, device="cuda")
    mean, rstd = (torch.empty(3000, device="cuda") for _ in range(2))
    y, dx, dw, db = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w), torch.empty_like(w)
    hb.layer_norm(x, w, None, y, mean, rstd)
    hb.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db)
    return dx, dw, db


def test_expired_wait_is_reported_once():
    assert hb.layer_norm_status() == 0
    _gradients()
    assert hb.layer_norm_status() == 0
    assert hb.lib().hilberta_selftest_layer_norm_timeout(None) == 0
    assert hb.layer_norm_status() == hb.ERR_TIMEOUT
    assert hb.layer_norm_status() == 0
    assert hb.packed_status() == 0   # flags of their own
    assert all(bool(torch.isfinite(t).all()) for t in _gradients())
    assert hb.layer_norm_status() == 0


def test_status_waits_for_work_on_other_streams():
    x, dy = (torch.randn((200000, 1024), device="cuda").bfloat16() for _ in range(2))
    mean, rstd = torch.zeros(200000, device="cuda"), torch.ones(200000, device="cuda")
    dx = torch.empty_like(x)
    side, done = torch.cuda.Stream(), torch.cuda.Event()
    hb.layer_norm_status()
    torch.cuda.synchronize()
    for _ in range(100):
        hb.layer_norm_backward(dy, x, None, mean, rstd, dx, None, None, stream=side)
    done.record(side)
    assert hb.layer_norm_status() == 0
    assert done.query()
