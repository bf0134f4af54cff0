"""Layer norm and its gradients against the formula in 64 bits and against differences.

Tolerances count roundings.  u = 2^-24 is half a step of fp32.  A sum of n terms in any order is off by at most
(n - 1) u times the sum of their magnitudes; over columns the kernel's chains are at most 32 + 16 long (a thread's
values, then lanes and warps), so 64 u bounds a mean with the roundings around it.  Outputs in bf16 add 2^-8."""
import numpy as np
import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
HALF = {torch.float32: U, torch.bfloat16: 2.0 ** -8}


def _reference(x, w, b, eps, unit):
    x = x.double()
    wide = lambda t: t.double().reshape(t.shape[:-1] + (1,) * (x.dim() - t.dim()) + t.shape[-1:])  # noqa: E731
    w = torch.ones(x.shape[-1], dtype=torch.float64, device=x.device) if w is None else wide(w) + (1 if unit else 0)
    b = 0 if b is None else wide(b)
    mean = x.mean(-1, keepdim=True)
    rstd = ((x - mean).square().mean(-1, keepdim=True) + eps).rsqrt()
    n = (x - mean) * rstd
    return n * w + b, mean.squeeze(-1), rstd.squeeze(-1), n, w


def _check_forward(x, w, b, eps=1e-6, unit=False, y=None):
    if y is None:
        y = torch.full_like(x, float("nan"))
    xs = x.clone()
    mean, rstd = (torch.full(x.shape[:-1], float("nan"), device="cuda") for _ in range(2))
    hb.layer_norm(x, w, b, y, mean, rstd, eps=eps, unit_offset=unit)
    ry, rm, rr, n, wd = _reference(xs, w, b, eps, unit)
    top = xs.double().abs().amax(-1)
    assert ((mean.double() - rm).abs() <= 64 * U * top).all()
    # the deviations carry the mean's error: relative to the standard deviation that is top * rstd
    worst = 64 * U * (1 + top * rr)
    assert ((rstd.double() / rr - 1).abs() <= 2 * worst).all()
    tol = (worst[..., None] * (1 + 2 * n.abs()) * wd.abs() + 4 * U * ry.abs()) + HALF[x.dtype] * ry.abs()
    if b is not None:
        tol = tol + 4 * U * (ry - n * wd).abs()
    assert ((y.double() - ry).abs() <= tol + 1e-30).all()
    return y, mean, rstd


def _make(shape, dtype, seed, offset=0.5, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    return (spread * torch.randn(shape, generator=g) + offset).to(dtype).cuda()


COLS = [1, 2, 7, 8, 63, 64, 65, 100, 256, 257, 512, 777, 1000, 1024, 1032, 1536, 2047, 2048, 4096, 4104, 5000, 8191, 8192, 16383, 16384]


@pytest.mark.parametrize("dtype,wdtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("cols", COLS)
def test_forward_and_gradients(cols, dtype, wdtype):
    for rows in (1, 5, 131):
        x = _make((rows, cols), dtype, cols + rows)
        w, b = _make((cols,), wdtype, 1, 1.0, 0.3), _make((cols,), wdtype, 2, 0.0, 0.3)
        _, mean, rstd = _check_forward(x, w, b)
        _check_backward(x, w, mean, rstd, _make((rows, cols), dtype, 3, 0.1, 1.0))


def _check_backward(x, w, mean, rstd, dy, unit=False, dx=None, which=(True, True, True), wlike=None):
    wlike = w if wlike is None else wlike
    dx = torch.full_like(x, float("nan")) if dx is None else dx
    dw, db = (torch.full_like(wlike, float("nan")) for _ in range(2))
    xs, gs = x.double(), dy.double()
    hb.layer_norm_backward(dy, x, w, mean, rstd, dx if which[0] else None, dw if which[1] else None, db if which[2] else None,
                           unit_offset=unit)
    n = (xs - mean.double()[..., None]) * rstd.double()[..., None]
    _, _, _, _, wd = _reference(xs, w, None, 0.0, unit)
    g = gs * wd
    r = rstd.double()[..., None]
    m1, m2 = g.mean(-1, keepdim=True), (g * n).mean(-1, keepdim=True)
    ref = r * (g - m1 - n * m2)
    size = g.abs() + g.abs().mean(-1, keepdim=True) + n.abs() * (g * n).abs().mean(-1, keepdim=True)
    # n itself: a subtraction and a product, relative to |x| + |mean|
    slip = 2 * U * (xs.abs() + mean.double().abs()[..., None]) * r
    slip_mean = (g.abs() * slip).mean(-1, keepdim=True)
    tol = r * (72 * U * size + slip * m2.abs() + n.abs() * slip_mean) + HALF[x.dtype] * ref.abs()
    if which[0]:
        assert ((dx.double() - ref).abs() <= tol + 1e-30).all()
    over = tuple(range(x.dim() - 1)) if wlike.dim() == 1 else tuple(range(1, x.dim() - 1))
    count = 1
    for a in over:
        count *= x.shape[a]
    for on, got, term, extra in ((which[1], dw, gs * n, gs.abs() * slip), (which[2], db, gs, 0 * gs)):
        if on:
            want = term.sum(over)
            tol = (count + 8) * U * term.abs().sum(over) + extra.sum(over) + HALF[wlike.dtype] * want.abs()
            assert ((got.double() - want).abs() <= tol + 1e-30).all()
    return dx, dw, db


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("B,S,cols", [(1, 3, 96), (2, 77, 1152), (5, 300, 130), (3, 1, 768), (300, 2, 64), (2, 2000, 512)])
def test_modulated_by_slices_of_one_tensor(B, S, cols, dtype):
    """One scale and shift per sample, read from (and their gradients written to) two slices of a wider tensor."""
    x, mod = _make((B, S, cols), dtype, 4), _make((B, 6 * cols), dtype, 5, 0.0, 0.5)
    shift, scale = mod[:, 2 * cols:3 * cols], mod[:, 3 * cols:4 * cols]
    y, mean, rstd = _check_forward(x, scale, shift, unit=True)
    dy = _make((B, S, cols), dtype, 6)
    dx, dw, db = _check_backward(x, scale, mean, rstd, dy, unit=True)
    dmod = torch.full_like(mod, 7.0)
    hb.layer_norm_backward(dy, x, scale, mean, rstd, dx, dmod[:, 3 * cols:4 * cols], dmod[:, 2 * cols:3 * cols], unit_offset=True)
    assert torch.equal(dmod[:, 3 * cols:4 * cols], dw) and torch.equal(dmod[:, 2 * cols:3 * cols], db)
    rest = torch.cat((dmod[:, :2 * cols], dmod[:, 4 * cols:]), 1)
    assert (rest == 7.0).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols,width,shift", [(64, 200, 8), (64, 201, 3), (1000, 2000, 1), (96, 1000, 500)])
def test_strided_and_misaligned_rows(cols, width, shift, dtype):
    rows = 37
    big, out = _make((rows, width), dtype, 7), torch.full((rows, width), 9.0, dtype=dtype, device="cuda")
    x, y = big[:, shift:shift + cols], out[:, shift:shift + cols]
    w, b = _make((cols,), dtype, 8, 1.0), _make((cols,), dtype, 9)
    _, mean, rstd = _check_forward(x, w, b, y=y)
    g = torch.full((rows, width), 9.0, dtype=dtype, device="cuda")
    _check_backward(x, w, mean, rstd, _make((rows, width), dtype, 10)[:, shift:shift + cols], dx=g[:, shift:shift + cols])
    for t in (out, g):
        rest = torch.cat((t[:, :shift], t[:, shift + cols:]), 1)
        assert (rest == 9.0).all()


@pytest.mark.parametrize("which", [(True, False, False), (False, True, False), (False, False, True), (True, True, False), (False, True, True)])
@pytest.mark.parametrize("rows", [3, 2500])
def test_each_gradient_alone_and_without_weights(which, rows):
    x, dy = _make((rows, 320), torch.bfloat16, 11), _make((rows, 320), torch.bfloat16, 12)
    w = _make((320,), torch.float32, 13)
    _, mean, rstd = _check_forward(x, None, None)
    _check_backward(x, None, mean, rstd, dy, which=which, wlike=w)
    _check_backward(x, w, mean, rstd, dy, which=which)


def test_in_place():
    for dtype, cols in ((torch.bfloat16, 1536), (torch.float32, 333), (torch.bfloat16, 12000)):
        x, w, b = _make((50, cols), dtype, 14), _make((cols,), dtype, 15), _make((cols,), dtype, 16)
        y, mean, rstd = _check_forward(x, w, b)
        z = x.clone()
        hb.layer_norm(z, w, b, z)
        assert torch.equal(z, y)
        dy = _make((50, cols), dtype, 17)
        dx, dw, db = _check_backward(x, w, mean, rstd, dy)
        for which in (0, 1):
            a, g = x.clone(), dy.clone()
            to = (a, g)[which]
            dw2, db2 = torch.empty_like(dw), torch.empty_like(db)
            hb.layer_norm_backward(g, a, w, mean, rstd, to, dw2, db2)
            assert torch.equal(to, dx) and torch.equal(dw2, dw) and torch.equal(db2, db)


def test_hard_rows():
    """Constant rows, rows far from zero, huge and tiny ones, and rows with infinities or NaN, which stay their own."""
    x = _make((8, 512), torch.float32, 18)
    x[0] = 3.25
    x[1] += 4096.0
    x[2] *= 1e15
    x[3] *= 1e-15
    y, mean, rstd = _check_forward(x, None, None)
    assert (y[0] == 0).all()
    bad = x.clone()
    bad[4, 100] = float("inf")
    bad[6, 5] = float("nan")
    z = torch.empty_like(bad)
    hb.layer_norm(bad, None, None, z)
    keep = [0, 1, 2, 3, 5, 7]
    assert torch.equal(z[keep], y[keep]) and z[[4, 6]].isnan().all()
    dx = torch.empty_like(bad)
    m, r = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
    hb.layer_norm(bad, None, None, z, m, r)
    dy = _make((8, 512), torch.float32, 19)
    ref = torch.empty_like(dx)
    hb.layer_norm_backward(dy, x, None, mean, rstd, ref, None, None)
    hb.layer_norm_backward(dy, bad, None, m, r, dx, None, None)
    assert torch.equal(dx[keep], ref[keep])


def test_no_rows():
    x, w = torch.empty((0, 64), device="cuda"), torch.ones(64, device="cuda")
    hb.layer_norm(x, w, w, torch.empty_like(x))
    dw, db = torch.full_like(w, 5.0), torch.full_like(w, 5.0)
    e = torch.empty(0, device="cuda")
    hb.layer_norm_backward(x, x, w, e, e, torch.empty_like(x), dw, db)
    assert (dw == 0).all() and (db == 0).all()


def test_gradients_against_differences():
    """Central differences of the forward formula in 64 bits: their own error is about h^2 and 1e-16 / h."""
    g = torch.Generator().manual_seed(20)
    B, S, C, eps, h = 2, 3, 10, 1e-3, 1e-5
    x, w, b, dy = (torch.randn(s, generator=g, dtype=torch.float64).float().double() for s in ((B, S, C), (B, C), (B, C), (B, S, C)))
    loss = lambda x, w, b: float((_reference(x, w, b, eps, True)[0] * dy).sum())  # noqa: E731
    xd, wd, bd, gd = (t.float().cuda() for t in (x, w, b, dy))
    y, mean, rstd = torch.empty_like(xd), torch.empty((B, S), device="cuda"), torch.empty((B, S), device="cuda")
    hb.layer_norm(xd, wd, bd, y, mean, rstd, eps=eps, unit_offset=True)
    grads = (torch.empty_like(xd), torch.empty_like(wd), torch.empty_like(bd))
    hb.layer_norm_backward(gd, xd, wd, mean, rstd, *grads, unit_offset=True)
    for k, got in enumerate(grads):
        args = [x, w, b]
        flat = got.cpu().double().flatten()
        for i in range(flat.numel()):
            d = torch.zeros_like(args[k]).flatten()
            d[i] = h
            d = d.view_as(args[k])
            up, down = list(args), list(args)
            up[k], down[k] = args[k] + d, args[k] - d
            assert abs((loss(*up) - loss(*down)) / (2 * h) - float(flat[i])) <= 2e-5


@pytest.mark.parametrize("rows,cols", [(3000, 256), (700, 1536), (64, 8192), (333, 777)])
def test_same_bits_again_on_other_streams_and_from_a_graph(rows, cols):
    x, dy = _make((rows, cols), torch.bfloat16, 21), _make((rows, cols), torch.bfloat16, 22)
    w, b = _make((cols,), torch.bfloat16, 23), _make((cols,), torch.bfloat16, 24)
    y, mean, rstd, dx = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda"), torch.empty_like(x)
    dw, db = torch.empty_like(w), torch.empty_like(w)
    outs = (y, mean, rstd, dx, dw, db)

    def step(stream=None):
        hb.layer_norm(x, w, b, y, mean, rstd, stream=stream)
        hb.layer_norm_backward(dy, x, w, mean, rstd, dx, dw, db, stream=stream)

    def wipe():
        for t in outs:
            t.fill_(float("nan"))
        torch.cuda.synchronize()

    step()
    torch.cuda.synchronize()
    first = [t.clone() for t in outs]
    side = torch.cuda.Stream()
    wipe()
    step(side)
    side.synchronize()
    assert all(torch.equal(a, t) for a, t in zip(first, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for k in range(2):
        x.copy_(_make((rows, cols), torch.bfloat16, 30 + k))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        wipe()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, t) for a, t in zip(want, outs))


def test_two_streams_at_once():
    a = [(_make((2000, 640), torch.bfloat16, 40 + k), _make((2000, 640), torch.bfloat16, 50 + k)) for k in range(2)]
    w = _make((640,), torch.float32, 60)
    stats, want = [], []
    for x, dy in a:
        _, mean, rstd = _check_forward(x, w, None)
        stats.append((mean, rstd))
        want.append([t.clone() for t in _check_backward(x, w, mean, rstd, dy)])
    streams = [torch.cuda.Stream() for _ in a]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [[torch.empty_like(t) for t in ts] for ts in want]
        torch.cuda.synchronize()
        for (x, dy), (mean, rstd), o, s in zip(a, stats, got, streams):
            hb.layer_norm_backward(dy, x, w, mean, rstd, *o, stream=s)
        torch.cuda.synchronize()
        for g, r in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(g, r))


def test_refusals():
    x, w = torch.ones((4, 64), device="cuda"), torch.ones(64, device="cuda")
    y, s = torch.empty_like(x), torch.empty(4, device="cuda")
    with pytest.raises(ValueError):
        hb.layer_norm(x, w, None, torch.empty((4, 63), device="cuda"))
    with pytest.raises(ValueError):
        hb.layer_norm(x, torch.ones(63, device="cuda"), None, y)
    with pytest.raises(ValueError):
        hb.layer_norm(x, w, torch.ones((4, 64), device="cuda"), y)
    with pytest.raises(ValueError):
        hb.layer_norm(x.t(), w, None, y)
    with pytest.raises(TypeError):
        hb.layer_norm(x, w, None, y, mean=s.double())
    with pytest.raises(ValueError):
        hb.layer_norm(x, w, None, y, mean=s.bfloat16())
    with pytest.raises(ValueError):
        hb.layer_norm(x, w.cpu(), None, y)
    with pytest.raises(ValueError):
        hb.layer_norm_backward(x, x, w, None, s, y, None, None)
    buf = torch.ones((5, 64), device="cuda")
    with pytest.raises(hb.HilbertaError):   # shifted by a row: neither apart nor in place
        hb.layer_norm(buf[:4], w, None, buf[1:])
    big = torch.ones((4000, 64), device="cuda")
    m = torch.empty(4000, device="cuda")
    with pytest.raises(hb.HilbertaError) as e:
        hb.layer_norm_backward(big, big, w, m, m, None, torch.empty_like(w), None, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == hb.ERR_BUFFER
    n = hb.layer_norm_workspace(big, w)
    assert n > 0
    hb.layer_norm(big, w, None, torch.empty_like(big), m, m.clone())
    hb.layer_norm_backward(big, big, w, m, m, None, torch.empty_like(w), None, workspace=torch.empty(n, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [64, 200, 1001, 1024])
def test_broadcast_rows(cols, dtype):
    x, dy, w = _make((37, cols), dtype, 40), _make((1, cols), dtype, 41), _make((cols,), dtype, 42)
    y, mean, rstd = _check_forward(x[:1].expand(37, cols), w, None, y=torch.empty_like(x))
    assert (y == y[0]).all()
    _check_backward(x[:1].expand(37, cols), w, mean, rstd, dy.expand(37, cols), dx=torch.empty_like(x))
    _, mean, rstd = _check_forward(x, w, None)
    _check_backward(x, w, mean, rstd, dy.expand(37, cols), dx=torch.empty_like(x))
    for out in (x[:1].expand(37, cols), torch.zeros(40 * cols, dtype=dtype, device="cuda").as_strided((37, cols), (cols // 2, 1))):
        with pytest.raises(hb.HilbertaError) as e:
            hb.layer_norm(y, w, None, out)
        assert e.value.status == hb.ERR_INVALID


def test_no_rows_in_several_groups():
    x, w, e = torch.empty((3, 0, 64), device="cuda"), torch.ones((3, 64), device="cuda"), torch.empty((3, 0), device="cuda")
    both = torch.full((3, 128), 5.0, device="cuda")
    hb.layer_norm_backward(x, x, w, e, e, None, both[:, :64], None)
    assert (both[:, :64] == 0).all() and (both[:, 64:] == 5).all()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    hb.layer_norm_backward(x, x, w, e, e, None, both[:, :64], both[:, 64:], stream=side)
    side.synchronize()
    assert (both == 0).all()
    none = torch.empty((0, 5, 64), device="cuda")
    hb.layer_norm_backward(none, none, None, e, e, None, both[:0, :64], both[:0, 64:])


@pytest.mark.parametrize("dtype,wdtype", [(torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32), (torch.float32, torch.float32)])
@pytest.mark.parametrize("cols", [8193, 8200, 8320, 10001, 10240, 11000, 12284, 12288, 14000, 15001, 16000, 16376])
def test_wide_rows(cols, dtype, wdtype):
    for rows in (1, 4, 331):
        x, w = _make((rows, cols), dtype, cols + rows), _make((cols,), wdtype, 1, 1.0, 0.3)
        _, mean, rstd = _check_forward(x, w, None)
        dy = _make((rows, cols), dtype, 3, 0.1, 1.0)
        _check_backward(x, w, mean, rstd, dy)
        _check_backward(x, None, mean, rstd, dy, wlike=w)


def test_wide_rows_in_groups_and_slices():
    cols = 9000
    x, mod = _make((3, 40, cols), torch.bfloat16, 50), _make((3, 2 * cols), torch.bfloat16, 51, 0.0, 0.3)
    _, mean, rstd = _check_forward(x, mod[:, :cols], mod[:, cols:], unit=True)
    _check_backward(x, mod[:, :cols], mean, rstd, _make((3, 40, cols), torch.bfloat16, 52), unit=True)
    big = _make((40, 2 * cols + 3), torch.bfloat16, 53)
    _, mean, rstd = _check_forward(big[:, 3:3 + cols], mod[0, :cols], None, y=torch.empty((40, cols), dtype=torch.bfloat16, device="cuda"))
    _check_backward(big[:, 3:3 + cols], mod[0, :cols], mean, rstd, big[:, cols:2 * cols], dx=torch.empty((40, cols), dtype=torch.bfloat16, device="cuda"))
