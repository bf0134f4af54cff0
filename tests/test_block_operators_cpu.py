"""Refusals and host arithmetic of the operators around the attention: no device is needed for either."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from paper_2509_26538_b200 import build

PTR = 1 << 20   # stands for a device pointer: every call here is refused before anything reads it


@pytest.fixture(scope="module")
def lib():
    build.build_library()
    return hb.lib()


def _norm(lib, x=PTR, w=PTR, b=None, y=2 * PTR, mean=None, rstd=None, rows=4, cols=64, per=0, sx=64, sy=64, sw=0, dtype=hb.BF16,
          wdtype=hb.BF16, eps=1e-6):
    return lib.hilberta_layer_norm(x, w, b, y, mean, rstd, rows, cols, per, sx, sy, sw, dtype, wdtype, 0, eps, None)


@pytest.mark.parametrize("bad,status", [
    (dict(x=None), hb.ERR_INVALID), (dict(y=None), hb.ERR_INVALID), (dict(rows=-1), hb.ERR_INVALID), (dict(cols=0), hb.ERR_INVALID),
    (dict(cols=16385, sx=16385, sy=16385), hb.ERR_UNSUPPORTED), (dict(per=-1), hb.ERR_INVALID), (dict(sx=-64), hb.ERR_INVALID),
    (dict(sy=63), hb.ERR_INVALID), (dict(eps=-1.0), hb.ERR_INVALID), (dict(eps=float("nan")), hb.ERR_INVALID),
    (dict(dtype=hb.FP8_E4M3, wdtype=hb.FP8_E4M3), hb.ERR_UNSUPPORTED), (dict(dtype=hb.FP32, wdtype=hb.BF16), hb.ERR_UNSUPPORTED),
    (dict(dtype=7), hb.ERR_INVALID), (dict(x=PTR + 1), hb.ERR_INVALID), (dict(w=PTR + 1), hb.ERR_INVALID), (dict(mean=PTR + 2), hb.ERR_INVALID),
    (dict(y=PTR + 128), hb.ERR_INVALID), (dict(per=2, sw=-64), hb.ERR_INVALID),
])
def test_layer_norm_refuses(lib, bad, status):
    assert _norm(lib, **bad) == status


def _norm_grad(lib, dy=1 << 35, x=1 << 30, w=PTR, mean=PTR, rstd=PTR, dx=1 << 40, dw=4 * PTR, db=5 * PTR, ws=None, ws_bytes=0, rows=4, cols=64,
               per=0, sdy=64, sx=64, sdx=64, sw=0, sdw=0, dtype=hb.BF16, wdtype=hb.FP32):
    return lib.hilberta_layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, ws, ws_bytes, rows, cols, per, sdy, sx, sdx, sw, sdw,
                                            dtype, wdtype, 0, None)


@pytest.mark.parametrize("bad,status", [
    (dict(dy=None), hb.ERR_INVALID), (dict(mean=None), hb.ERR_INVALID), (dict(rstd=None), hb.ERR_INVALID),
    (dict(dx=None, dw=None, db=None), hb.ERR_INVALID), (dict(sdx=60), hb.ERR_INVALID), (dict(per=2, sw=0, sdw=63), hb.ERR_INVALID),
    (dict(dx=(1 << 30) + 64), hb.ERR_INVALID), (dict(rows=70000, per=1, sdw=64), hb.ERR_UNSUPPORTED), (dict(dw=4 * PTR + 2), hb.ERR_INVALID),
    (dict(cols=20000, sdy=20000, sx=20000, sdx=20000), hb.ERR_UNSUPPORTED),
])
def test_layer_norm_backward_refuses(lib, bad, status):
    assert _norm_grad(lib, **bad) == status


@pytest.mark.parametrize("bad", [
    dict(dw=4 * PTR, db=4 * PTR), dict(dw=4 * PTR, db=4 * PTR + 252), dict(per=2, dw=4 * PTR, db=4 * PTR + 128, sdw=96),
    dict(per=2, dw=4 * PTR + 256, db=4 * PTR, sdw=64), dict(per=1, sdw=128, dw=4 * PTR + 3 * 512 + 4, db=4 * PTR),
])
def test_layer_norm_backward_refuses_gradients_that_overlap(lib, bad):
    assert _norm_grad(lib, **{"ws": PTR, "ws_bytes": 1 << 30, **bad}) == hb.ERR_INVALID


def test_layer_norm_backward_takes_gradients_side_by_side(lib):
    if torch.cuda.is_available():
        pytest.skip("would launch on made-up pointers")
    for ok in (dict(dw=4 * PTR, db=4 * PTR + 256), dict(per=2, dw=4 * PTR + 256, db=4 * PTR, sdw=128), dict(per=1, sdw=192, dw=4 * PTR, db=4 * PTR + 512)):
        assert _norm_grad(lib, ws=PTR, ws_bytes=1 << 30, **ok) == hb.ERR_CUDA


def test_statistics_have_a_place_each(lib):
    assert _norm(lib, mean=PTR, rstd=PTR) == hb.ERR_INVALID


def _rotary(lib, fn="hilberta_rotary", x=PTR, out=2 * PTR, pos=None, freq=None, axis=None, pairs=32, axes=1, factor=1.0, plan=None, batch=1,
            heads=2, S=5, dim=64, dtype=hb.BF16, strides=(640, 320, 64, 640, 320, 64), no_freq=False):
    f = np.ones(max(pairs, 1)) if freq is None else np.asarray(freq, dtype=np.float64)
    a = None if axis is None else np.asarray(axis, dtype=np.int32)
    st = None if strides is None else (ctypes.c_int64 * 6)(*strides)
    return getattr(lib, fn)(x, out, pos, None if no_freq else f.ctypes.data, None if a is None else a.ctypes.data, pairs, axes, 0, factor,
                            plan, batch, heads, S, dim, dtype, st, 0, None)


@pytest.mark.parametrize("fn", ["hilberta_rotary", "hilberta_rotary_backward"])
@pytest.mark.parametrize("bad,status", [
    (dict(x=None), hb.ERR_INVALID), (dict(out=None), hb.ERR_INVALID), (dict(no_freq=True), hb.ERR_INVALID), (dict(strides=None), hb.ERR_INVALID),
    (dict(pairs=0), hb.ERR_INVALID), (dict(pairs=33), hb.ERR_INVALID), (dict(axes=0), hb.ERR_INVALID), (dict(axes=2), hb.ERR_INVALID),
    (dict(pos=PTR, axes=2, axis=[2] * 32), hb.ERR_INVALID), (dict(pos=PTR, axes=17, axis=[0] * 32), hb.ERR_UNSUPPORTED),
    (dict(pos=PTR + 2), hb.ERR_INVALID), (dict(freq=[np.inf] * 32), hb.ERR_INVALID), (dict(factor=float("nan")), hb.ERR_INVALID),
    (dict(dim=300, pairs=40), hb.ERR_UNSUPPORTED), (dict(dtype=hb.FP8_E4M3), hb.ERR_UNSUPPORTED), (dict(dtype=5), hb.ERR_INVALID),
    (dict(batch=-1), hb.ERR_INVALID), (dict(heads=0), hb.ERR_INVALID), (dict(S=-1), hb.ERR_INVALID), (dict(x=PTR + 1), hb.ERR_INVALID),
    (dict(batch=1 << 20, S=1 << 12), hb.ERR_UNSUPPORTED), (dict(strides=(640, 320, -64, 640, 320, 64)), hb.ERR_INVALID),
    (dict(strides=(640, 320, 64, 640, 320, 0)), hb.ERR_INVALID),
])
def test_rotary_refuses(lib, fn, bad, status):
    assert _rotary(lib, fn, **bad) == status


def test_rotary_frequencies():
    j = np.arange(32)
    plain = 500000.0 ** (-j / 32)
    f, factor = hb.rotary_frequencies(32, base=500000.0)
    assert factor == 1.0 and np.allclose(f.numpy(), plain, rtol=1e-14, atol=0)
    f, factor = hb.rotary_frequencies(32, base=500000.0, scaling=hb.ROTARY_LINEAR, scale=8.0)
    assert factor == 1.0 and np.allclose(f.numpy(), plain / 8, rtol=1e-14, atol=0)
    f, factor = hb.rotary_frequencies(32, base=500000.0, scaling=hb.ROTARY_BASE, scale=8.0)
    assert factor == 1.0 and f[0] == 1.0 and np.isclose(f[-1], plain[-1] / 8, rtol=1e-13)
    f, factor = hb.rotary_frequencies(32, base=500000.0, scaling=hb.ROTARY_BANDS, scale=8.0, context=8192.0, slow=1.0, fast=4.0)
    turns = 8192 * plain / (2 * math.pi)
    assert np.isclose(factor, 1 + 0.1 * math.log(8.0), rtol=1e-15)
    assert np.allclose(f.numpy()[turns > 4], plain[turns > 4], rtol=1e-14, atol=0)
    assert np.allclose(f.numpy()[turns < 1], plain[turns < 1] / 8, rtol=1e-14, atol=0)
    mid = (turns > 1) & (turns < 4)
    ramp = (turns[mid] - 1) / 3
    assert mid.any() and np.allclose(f.numpy()[mid], plain[mid] * (ramp + (1 - ramp) / 8), rtol=1e-12, atol=0)
    f, _ = hb.rotary_frequencies(1, scaling=hb.ROTARY_BASE, scale=2.0)
    assert f.tolist() == [1.0]


@pytest.mark.parametrize("bad", [dict(pairs=0), dict(base=0.0), dict(base=float("inf")), dict(scaling=4), dict(scaling=-1),
                                 dict(scaling=hb.ROTARY_LINEAR, scale=0.5), dict(scaling=hb.ROTARY_LINEAR, scale=float("nan")),
                                 dict(scaling=hb.ROTARY_BANDS, scale=2.0, context=0.0),
                                 dict(scaling=hb.ROTARY_BANDS, scale=2.0, context=4096.0, slow=4.0, fast=4.0),
                                 dict(scaling=hb.ROTARY_BANDS, scale=2.0, context=4096.0, slow=-1.0)])
def test_rotary_frequencies_refuses(bad):
    with pytest.raises(hb.HilbertaError) as e:
        hb.rotary_frequencies(**{"pairs": 8, **bad})
    assert e.value.status == hb.ERR_INVALID


def test_binding_refuses_shapes_before_the_library():
    x = torch.zeros((2, 3, 8))
    assert hb._row_stride(x, "x") == 8 and hb._row_stride(x[:, :, :4], "x") == 8 and hb._row_stride(x[:1, :, 2:], "x") == 8
    for bad in (x.transpose(0, 2), x[:, :2], x.permute(1, 0, 2)):
        with pytest.raises(ValueError):
            hb._row_stride(bad, "x")
    with pytest.raises(ValueError):
        hb._norm_weights(x, torch.zeros(3, 8), None)
    assert hb._norm_weights(x, None, None) == (0, 0, hb.FP32)
    assert hb._norm_weights(x, torch.zeros(2, 16)[:, 8:], None) == (3, 16, hb.FP32)
    with pytest.raises(ValueError):
        hb._norm_weights(x, torch.zeros(8), torch.zeros(8).bfloat16())
    with pytest.raises(ValueError):
        hb._norm_weights(x, torch.zeros(2, 8), torch.zeros(2, 16)[:, 8:])


def _packed(lib, fn="hilberta_packed_forward", q=1 << 30, k=1 << 31, v=1 << 32, out=1 << 33, lse=None, cu=PTR, n=1, total=10, heads=4, kv=2,
            dim=64, dtype=hb.BF16, st=(256, 64, 128, 64, 128, 64, 256, 64), scale=0.0):
    strides = None if st is None else (ctypes.c_int64 * 8)(*st)
    return lib.hilberta_packed_forward(q, k, v, out, lse, cu, n, total, heads, kv, dim, dtype, strides, 1, scale, None)


BAD_PACKED = [
    (dict(q=None), hb.ERR_INVALID), (dict(k=None), hb.ERR_INVALID), (dict(v=None), hb.ERR_INVALID), (dict(out=None), hb.ERR_INVALID),
    (dict(cu=None), hb.ERR_INVALID), (dict(st=None), hb.ERR_INVALID), (dict(n=-1), hb.ERR_INVALID), (dict(total=-1), hb.ERR_INVALID),
    (dict(heads=0), hb.ERR_INVALID), (dict(kv=0), hb.ERR_INVALID), (dict(kv=3), hb.ERR_INVALID), (dict(dim=0), hb.ERR_INVALID),
    (dict(dim=96), hb.ERR_UNSUPPORTED), (dict(dtype=hb.FP32), hb.ERR_UNSUPPORTED), (dict(dtype=hb.FP8_E4M3), hb.ERR_UNSUPPORTED),
    (dict(dtype=9), hb.ERR_INVALID), (dict(n=65537), hb.ERR_UNSUPPORTED), (dict(total=(1 << 26) + 1), hb.ERR_UNSUPPORTED),
    (dict(q=(1 << 30) + 8), hb.ERR_INVALID), (dict(lse=PTR + 1), hb.ERR_INVALID), (dict(cu=PTR + 2), hb.ERR_INVALID),
    (dict(st=(256, 60, 128, 64, 128, 64, 256, 64)), hb.ERR_INVALID), (dict(st=(256, 64, 0, 64, 128, 64, 256, 64)), hb.ERR_INVALID),
    (dict(st=(256, 64, 128, 64, -128, 64, 256, 64)), hb.ERR_INVALID), (dict(scale=float("nan")), hb.ERR_INVALID),
    (dict(out=1 << 30), hb.ERR_INVALID), (dict(out=(1 << 31) + 128), hb.ERR_INVALID),
]


@pytest.mark.parametrize("bad,status", BAD_PACKED)
def test_packed_forward_refuses(lib, bad, status):
    assert _packed(lib, **bad) == status


def _packed_grad(lib, ptrs=None, lse=PTR, ws=PTR, ws_bytes=320, cu=PTR, n=1, total=10, heads=4, kv=2, dim=64, dtype=hb.BF16, st=None, scale=0.0):
    p = [(i + 1) << 30 for i in range(8)]
    for i, x in (ptrs or {}).items():
        p[i] = x
    q, k = (256, 64), (128, 64)
    strides = (ctypes.c_int64 * 16)(*(st or q + q + k + k + q + q + k + k))
    return lib.hilberta_packed_backward(*p[:5], lse, *p[5:], ws, ws_bytes, cu, n, total, heads, kv, dim, dtype, strides, 1, scale, None)


@pytest.mark.parametrize("bad,status", [(dict(ptrs={i: None}), hb.ERR_INVALID) for i in range(8)] + [
    (dict(lse=None), hb.ERR_INVALID), (dict(ws=None), hb.ERR_BUFFER), (dict(ws_bytes=319), hb.ERR_BUFFER), (dict(ws=PTR + 8), hb.ERR_INVALID),
    (dict(ptrs={5: 1 << 30}), hb.ERR_INVALID), (dict(ptrs={6: (7 << 30) + 64, 7: 7 << 30}), hb.ERR_INVALID), (dict(kv=3), hb.ERR_INVALID),
    (dict(dim=32), hb.ERR_UNSUPPORTED), (dict(dtype=hb.FP32), hb.ERR_UNSUPPORTED), (dict(scale=float("nan")), hb.ERR_INVALID),
])
def test_packed_backward_refuses(lib, bad, status):
    assert _packed_grad(lib, **bad) == status


def test_slices_of_one_buffer_pass_the_overlap_test(lib):
    """q, k, v and out side by side within a token, or head by head: accepted up to the point where a device is needed."""
    if torch.cuda.is_available():
        pytest.skip("would launch on made-up pointers")
    base = 1 << 30
    token = (4 + 2 + 2 + 4) * 64
    st = (token, 64) * 4
    ok = _packed(lib, q=base, k=base + 512, v=base + 768, out=base + 1024, st=st)
    assert ok == hb.ERR_CUDA
    assert _packed(lib, q=base, k=base + 512, v=base + 768, out=base + 1000 // 16 * 16, st=st) == hb.ERR_INVALID
    pairs = (1024, 128) * 4   # q and out interleaved head by head, one key head for each
    far = 1 << 40
    assert _packed(lib, q=base, k=far, v=far + (1 << 30), out=base + 128, kv=4, st=pairs) == hb.ERR_CUDA
    assert _packed(lib, q=base, k=far, v=far + (1 << 30), out=base + 112, kv=4, st=pairs) == hb.ERR_INVALID
    assert lib.hilberta_packed_workspace(10, 4) == 320 and lib.hilberta_packed_workspace(0, 4) == 0


def test_row_stride_of_broadcast_and_overlapping_rows():
    one, line = torch.zeros((1, 8)), torch.zeros(40)
    assert hb._row_stride(one.expand(4, 8), "x") == 0 and hb._row_stride(one.expand(2, 3, 8), "x") == 0
    assert hb._row_stride(line.as_strided((4, 8), (4, 1)), "x") == 4
    assert hb._row_stride(line.as_strided((1, 8), (4, 1)), "x") == 8   # one row has any stride
    with pytest.raises(ValueError):
        hb._row_stride(torch.zeros((2, 1, 8)).expand(2, 3, 8), "x")
