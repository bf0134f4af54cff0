"""Which places of rows the layer norm takes and which it refuses: exact for slices of one buffer.  No device is needed."""
import ctypes

import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from paper_2509_26538_b200 import build

BASE = 1 << 30


@pytest.fixture(scope="module")
def lib():
    if torch.cuda.is_available():
        pytest.skip("would launch on made-up pointers")
    build.build_library()
    return hb.lib()


def _norm(lib, y, rows=4, cols=64, sx=128, sy=128):
    return lib.hilberta_layer_norm(BASE, None, None, y, None, None, rows, cols, 0, sx, sy, 0, hb.BF16, hb.BF16, 0, ctypes.c_float(1e-6), None)


def _norm_grad(lib, dy, dx, rows=4, cols=64, stride=192, sdx=None):
    return lib.hilberta_layer_norm_backward(dy, BASE, None, 1 << 20, 1 << 20, dx, None, None, None, 0, rows, cols, 0, stride, stride,
                                            stride if sdx is None else sdx, 0, 0, hb.BF16, hb.BF16, 0, None)


# ERR_CUDA: every check is passed, and there is no device
@pytest.mark.parametrize("kw,status", [
    (dict(y=BASE + 128), hb.ERR_CUDA), (dict(y=BASE), hb.ERR_CUDA), (dict(y=BASE - 128), hb.ERR_CUDA), (dict(y=BASE + 128 + 3 * 256), hb.ERR_CUDA),
    (dict(y=BASE + 126), hb.ERR_INVALID), (dict(y=BASE + 130), hb.ERR_INVALID), (dict(y=BASE + 256), hb.ERR_INVALID), (dict(y=BASE - 126), hb.ERR_INVALID),
    (dict(y=BASE + 3 * 256 + 128), hb.ERR_CUDA), (dict(y=BASE + 3 * 256 + 126), hb.ERR_INVALID), (dict(y=BASE + 4 * 256 - 2), hb.ERR_CUDA),
    (dict(y=BASE + 128, sy=130), hb.ERR_INVALID), (dict(y=BASE + 128, sy=64), hb.ERR_INVALID), (dict(y=BASE + 2048, sy=64), hb.ERR_CUDA),
    # one row has any stride
    (dict(y=BASE, rows=1, sx=0, sy=64), hb.ERR_CUDA), (dict(y=BASE + 126, rows=1, sx=0, sy=64), hb.ERR_INVALID),
    (dict(y=BASE + 128, rows=1, sx=4096, sy=64), hb.ERR_CUDA), (dict(y=BASE, rows=0), hb.ERR_CUDA),
    # the same row for all of x
    (dict(y=BASE, sx=0, sy=64), hb.ERR_INVALID), (dict(y=BASE + 128, sx=0, sy=64), hb.ERR_CUDA),
])
def test_forward(lib, kw, status):
    assert _norm(lib, **kw) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dy=BASE + 128, dx=BASE + 256), hb.ERR_CUDA), (dict(dy=BASE + 128, dx=BASE), hb.ERR_CUDA), (dict(dy=BASE + 128, dx=BASE + 128), hb.ERR_CUDA),
    (dict(dy=BASE + 128, dx=BASE + 258), hb.ERR_INVALID), (dict(dy=BASE + 128, dx=BASE + 254), hb.ERR_INVALID),
    (dict(dy=BASE + 128, dx=BASE + 64), hb.ERR_INVALID), (dict(dy=BASE + 128, dx=BASE + 256, sdx=194), hb.ERR_INVALID),
])
def test_backward(lib, kw, status):
    assert _norm_grad(lib, **kw) == status
