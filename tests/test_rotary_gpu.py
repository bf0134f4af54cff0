"""Rotary positions and their gradient against the formula in 64 bits.

Tolerance: u = 2^-24.  The angle in turns is exact but for 2^-31 of half a turn and one rounding to fp32 of at most an
eighth of a turn (below u in radians), cosine and sine are Taylor series evaluated to two units in the last place (2 u), the factor's own
rounding and its product add 2 u, the two products and their sum 2 u of |a| + |b|: 8 u (|a| + |b|) factor covers it.
Outputs in bf16 add 2^-8 of the value.  Copied elements are the same bits."""
import math

import numpy as np
import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _reference(x, inv_freq, pos, axis, interleaved, factor, sign):
    """x [B, H, S, D] on the CPU; pos int64 [B, S, axes]."""
    P = inv_freq.numel()
    ax = torch.zeros(P, dtype=torch.long) if axis is None else axis.long()
    two_pi = np.longdouble("6.283185307179586476925286766559005768")
    t = pos[..., ax].numpy().astype(np.longdouble) * inv_freq.numpy().astype(np.longdouble)
    t = np.fmod(t, two_pi).astype(np.float64)
    cos, sin = (torch.from_numpy(f(t))[:, None] * factor for f in (np.cos, np.sin))
    sin = sin * sign
    x = x.double()
    i = torch.arange(P)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + P)
    out, tol = x.clone(), torch.zeros_like(x)
    out[..., a] = x[..., a] * cos - x[..., b] * sin
    out[..., b] = x[..., a] * sin + x[..., b] * cos
    tol[..., a] = tol[..., b] = 8 * U * abs(factor) * (x[..., a].abs() + x[..., b].abs())
    return out, tol


def _check(x, inv_freq, positions=None, axis=None, interleaved=False, factor=1.0, plan=None, out=None, back=False):
    B, H, S, D = x.shape
    xs = x.cpu().clone()
    if positions is None:
        pos = torch.arange(S).expand(B, S)[..., None]
    else:
        pos = positions.cpu().long()
        pos = pos if axis is not None else pos[..., None]
        pos = pos.expand(B, S, pos.shape[-1])
    out = torch.full_like(x, float("nan")) if out is None else out
    fn = hb.rotary_backward if back else hb.rotary
    fn(x, out, inv_freq, positions, axis=axis, interleaved=interleaved, factor=factor, plan=plan)
    if plan is not None:
        table = torch.from_numpy(plan.export(hb.EXPORT_ORIG2PHYS if back else hb.EXPORT_PHYS2ORIG)).long()
        xs = xs[:, :, table]
        if not back:
            pos = pos[:, table]
    ref, tol = _reference(xs, inv_freq, pos, axis, interleaved, factor, -1.0 if back else 1.0)
    got = out.cpu()
    err = (got.double() - ref).abs()
    assert (err <= tol + (2.0 ** -8 if x.dtype == torch.bfloat16 else 0.0) * ref.abs() + 1e-38).all()
    P = inv_freq.numel()
    assert torch.equal(got[..., 2 * P:], xs[..., 2 * P:])
    return out


def _make(shape, dtype, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


DIMS = [(2, 1), (32, 16), (64, 32), (64, 5), (64, 8), (80, 24), (96, 36), (100, 50), (128, 64), (128, 1), (192, 96), (250, 125), (256, 128), (256, 100)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", DIMS)
def test_forward_and_gradient(dim, pairs, interleaved, dtype):
    for B, H, S in ((1, 1, 1), (2, 3, 37), (1, 9, 130)):
        x = _make((B, H, S, dim), dtype, dim + pairs + S)
        f, factor = hb.rotary_frequencies(pairs)
        _check(x, f, interleaved=interleaved)
        pos = torch.randint(-2 ** 31, 2 ** 31 - 1, (B, S), generator=torch.Generator().manual_seed(S)).int().cuda()
        _check(x, f, pos, interleaved=interleaved, factor=1.25, back=True)


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", [(128, 64), (72, 20), (66, 33)])
def test_turning_back_restores(dim, pairs, interleaved):
    x = _make((2, 5, 40, dim), torch.float32, 1)
    f, _ = hb.rotary_frequencies(pairs)
    y, z = torch.empty_like(x), torch.empty_like(x)
    hb.rotary(x, y, f, interleaved=interleaved)
    hb.rotary_backward(y, z, f, interleaved=interleaved)
    assert ((z - x).abs() <= 32 * U * (x.abs().amax(-1, keepdim=True))).all()


def test_gradient_is_the_transpose():
    """sum(rotary(x) dy) = sum(x rotary_backward(dy)), exactly bilinear: in fp32 to the sums' roundings."""
    x, dy = _make((2, 3, 50, 96), torch.float32, 2), _make((2, 3, 50, 96), torch.float32, 3)
    f, factor = hb.rotary_frequencies(40, scaling=hb.ROTARY_BANDS, scale=4.0, context=64.0)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    hb.rotary(x, y, f, factor=factor)
    hb.rotary_backward(dy, dx, f, factor=factor)
    a, b = (y.double() * dy.double()).sum(), (x.double() * dx.double()).sum()
    size = (x.double().abs().sum(-1) * dy.double().abs().sum(-1)).sum()
    assert abs(a - b) <= 32 * U * size


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("Hq,Hk,dim,pairs", [(4, 2, 64, 32), (3, 1, 80, 24), (6, 6, 100, 31)])
def test_slices_of_a_projection_in_place(Hq, Hk, dim, pairs, dtype):
    """q and k of a packed [tokens, heads, head_dim] projection turned in place in one call; v stays."""
    T = 53
    qkv = _make((1, T, Hq + 2 * Hk, dim), dtype, 4)
    was = qkv.clone()
    f, _ = hb.rotary_frequencies(pairs)
    pos = torch.cat([torch.arange(20), torch.arange(33)]).int().cuda()
    x = qkv.transpose(1, 2)[:, :Hq + Hk]
    ref = torch.empty((1, Hq + Hk, T, dim), dtype=dtype, device="cuda")
    _check(x, f, pos, out=ref)
    _check(x, f, pos, out=x)
    assert torch.equal(qkv.transpose(1, 2)[:, :Hq + Hk], ref)
    assert torch.equal(qkv[:, :, Hq + Hk:], was[:, :, Hq + Hk:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("H,W,text,B,heads,dim", [(8, 8, 0, 1, 1, 64), (16, 16, 5, 2, 3, 128), (12, 20, 7, 1, 4, 72)])
def test_with_a_plan_and_three_axes(H, W, text, B, heads, dim, interleaved, dtype):
    n = 1 << (max(H, W) - 1).bit_length()
    plan = hb.Plan(H, W, n * n // 4, 3, 2, text)
    try:
        S, P = plan.S, dim // 2
        pos = torch.zeros((S, 3), dtype=torch.int32)
        pos[:text, 0] = torch.arange(text)
        pos[text:, 1] = torch.arange(H * W) // W
        pos[text:, 2] = torch.arange(H * W) % W
        axis = torch.arange(P).remainder(3).sort().values.int()
        f, _ = hb.rotary_frequencies(P)
        x = _make((B, heads, S, dim), dtype, 5)
        y = _check(x, f, pos.cuda(), axis=axis, interleaved=interleaved, plan=plan)
        # the gather and the rotation one after the other: the same bits
        if dim * x.element_size() % 16 == 0:
            z, t = torch.empty_like(x), torch.empty_like(x)
            hb.rotary(x, t, f, pos.cuda(), axis=axis, interleaved=interleaved)
            plan.permute(t, z)
            assert torch.equal(z, y)
        _check(x, f, pos.cuda(), axis=axis, interleaved=interleaved, plan=plan, back=True)
    finally:
        plan.destroy()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,pairs", [(64, 21), (64, 24), (128, 50)])
def test_copied_elements_do_not_touch_the_rotated(dim, pairs, interleaved, dtype):
    x = _make((1, 2, 9, dim), dtype, 6)
    f, _ = hb.rotary_frequencies(pairs)
    y = _check(x, f, interleaved=interleaved)
    x[..., 2 * pairs::2] = float("nan")
    x[..., 2 * pairs + 1::2] = float("inf")
    z = torch.empty_like(x)
    hb.rotary(x, z, f, interleaved=interleaved)
    assert torch.equal(z[..., :2 * pairs], y[..., :2 * pairs])
    assert z[..., 2 * pairs::2].isnan().all() and (z[..., 2 * pairs + 1::2] == float("inf")).all()


def test_many_batch_items_and_heads():
    f, _ = hb.rotary_frequencies(16)
    x = _make((3000, 2, 1, 32), torch.bfloat16, 7)
    pos = torch.randint(0, 10 ** 6, (3000, 1), generator=torch.Generator().manual_seed(8)).int().cuda()
    _check(x, f, pos)
    _check(_make((2, 300, 3, 32), torch.bfloat16, 9), f)
    _check(_make((1, 20, 9000, 32), torch.bfloat16, 10), f, interleaved=True)
    e = torch.empty((0, 4, 5, 32), device="cuda")
    hb.rotary(e, e.clone(), f)


def test_offsets_beyond_32_bits():
    """A token stride that takes the last rows 2^32 elements away (8 GB of bf16 in a view)."""
    stride = 2 ** 31 // 3 // 8 * 8
    buf = torch.zeros(6 * stride + 128, dtype=torch.bfloat16, device="cuda")
    x = buf.as_strided((1, 2, 7, 64), (0, 64, stride, 1))
    x.copy_(_make((1, 2, 7, 64), torch.bfloat16, 11))
    out = torch.empty((1, 2, 7, 64), dtype=torch.bfloat16, device="cuda")
    f, _ = hb.rotary_frequencies(32)
    _check(x, f, out=out)
    _check(out, f, out=x)


@pytest.mark.parametrize("dim,pairs", [(128, 64), (90, 31)])
def test_other_streams_and_graphs(dim, pairs):
    x, f = _make((2, 4, 300, dim), torch.bfloat16, 12), hb.rotary_frequencies(pairs)[0]
    pos = torch.arange(300).int().cuda()
    y = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    hb.rotary(x, y, f, pos, stream=side)
    side.synchronize()
    ref = _check(x, f, pos)
    assert torch.equal(y, ref)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hb.rotary(x, y, f, pos)
        hb.rotary_backward(y, y, f, pos)
        hb.rotary(y, y, f, pos)
    f.zero_()   # the frequencies were read by the call
    y.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert ((y.float() - ref.float()).abs() <= 3 * 2.0 ** -7 * x.float().abs().amax(-1, keepdim=True)).all()


def test_refusals():
    f, _ = hb.rotary_frequencies(32)
    x = torch.ones((1, 2, 5, 64), device="cuda")
    y = torch.empty_like(x)
    for bad in (dict(inv_freq=f.float()), dict(inv_freq=f.cuda()), dict(positions=torch.arange(5).cuda()), dict(positions=torch.arange(4).int().cuda()),
                dict(axis=torch.zeros(31, dtype=torch.int32)), dict(positions=torch.arange(5).int())):
        with pytest.raises(ValueError):
            hb.rotary(x, y, **{"inv_freq": f, **bad})
    with pytest.raises(ValueError):
        hb.rotary(x, y.half(), f)
    with pytest.raises(hb.HilbertaError):
        hb.rotary(x, y, torch.ones(33, dtype=torch.float64))
    with pytest.raises(hb.HilbertaError):
        hb.rotary(x, y, f, torch.zeros((5, 2), dtype=torch.int32, device="cuda"), axis=torch.full((32,), 2, dtype=torch.int32))
    with pytest.raises(hb.HilbertaError):
        hb.rotary(x, y, f * float("nan"))
    with pytest.raises(hb.HilbertaError):   # shifted by a token: neither apart nor in place
        buf = torch.ones((1, 2, 6, 64), device="cuda")
        hb.rotary(buf[:, :, :5], buf[:, :, 1:], f)
    plan = hb.Plan(2, 2, 2, 0, 0, 1)
    try:
        with pytest.raises(hb.HilbertaError):   # in place with a gather
            hb.rotary(x, x, f, plan=plan)
        with pytest.raises(hb.HilbertaError):
            hb.rotary(x[:, :, :4], y[:, :, :4], f, plan=plan)
        hb.rotary(x, y, f, plan=plan)
    finally:
        plan.destroy()
