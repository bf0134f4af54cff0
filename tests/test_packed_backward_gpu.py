"""Gradients of the attention over packed sequences against the formula in 64 bits and against differences.

Tolerances.  P and dS are rounded to bf16 before they are summed over queries or keys, and so is `out`, through which
delta is off by at most 2^-8 sum |dout out|: element errors of relative 2^-8 that add up with random signs.  The sums'
relative error in the 2-norm is then below 5e-3, the bound that the sparse gradients of this library are held to, from 64
tokens on (with fewer, dS is a small difference).  Per element: 2^-8 of the sum of the magnitudes that are added (P |dout|, |dS| |k| with |dS| taken as P (|dP| + |delta|)), twice
for the two roundings on the way (operands, delta), and the result's own 2^-8."""
import math

import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from test_packed_gpu import CANARY, LENS, make

pytestmark = pytest.mark.gpu


def _tensors(q, k, v, cu, causal, seed, scale=0.0):
    T, H, D = q.shape
    out, lse = torch.full((T, H, D), CANARY, dtype=torch.bfloat16, device="cuda"), torch.full((H, T), CANARY, device="cuda")
    hb.packed_forward(q, k, v, out, cu, lse=lse, causal=causal, scale=scale)
    dout = torch.randn((T, H, D), generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()
    return dout, out, lse


def _reference(dout, q, k, v, cu, causal, scale):
    """Per sequence: its rows, dq, dk, dv [n, heads, D] and the magnitudes their roundings are relative to, in 64 bits."""
    H, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    scale = scale or D ** -0.5
    bounds = cu.tolist()
    for a, b in zip(bounds, bounds[1:]):
        if b <= a:
            continue
        qs, ks, vs, gs = (t[a:b].double().transpose(0, 1) for t in (q, k, v, dout))
        ks, vs = (t.repeat_interleave(H // Hk, 0) for t in (ks, vs))
        s = qs @ ks.transpose(1, 2) * scale
        if causal:
            s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1), -math.inf)
        p = torch.softmax(s, -1)
        dp = gs @ vs.transpose(1, 2)
        delta = (p * dp).sum(-1, keepdim=True)
        ds = p * (dp - delta)
        # |delta| as it can be off: through |out| rounded
        size = p * (dp.abs() + (gs.abs() * (p @ vs).abs()).sum(-1, keepdim=True))
        fold = lambda t: t.unflatten(0, (Hk, H // Hk)).sum(1).transpose(0, 1)  # noqa: E731
        flat = lambda t: t.transpose(0, 1)  # noqa: E731
        yield (a, b, (flat(ds @ ks) * scale, fold(ds.transpose(1, 2) @ qs) * scale, fold(p.transpose(1, 2) @ gs)),
               (flat(size @ ks.abs()) * scale, fold(size.transpose(1, 2) @ qs.abs()) * scale, fold(p.transpose(1, 2) @ gs.abs())))


def _check(q, k, v, cu, causal, seed=1, scale=0.0, grads=None):
    dout, out, lse = _tensors(q, k, v, cu, causal, seed, scale)
    if grads is None:
        grads = [torch.full(t.shape, CANARY, dtype=torch.bfloat16, device="cuda") for t in (q, k, v)]
    hb.packed_backward(dout, q, k, v, out, lse, *grads, cu, causal=causal, scale=scale)
    assert hb.packed_status() == 0
    mine = torch.zeros(q.shape[0], dtype=torch.bool, device="cuda")
    for a, b, want, size in _reference(dout, q, k, v, cu, causal, scale):
        mine[a:b] = True
        for name, g, w, m in zip(("dq", "dk", "dv"), grads, want, size):
            err = (g[a:b].double() - w).abs()
            assert (err <= 2.0 ** -8 * (2 * m + w.abs()) + 1e-30).all(), (name, a, b, float((err / m).max()))
            if b - a == 1 and name != "dv":
                assert (g[a:b] == 0).all(), name   # one key: a weight of one, whatever the scores
            elif b - a >= 64:
                assert float(err.norm() / w.norm()) <= 5e-3, (name, a, b, float(err.norm() / w.norm()))
    for g in grads:
        assert (g[~mine] == CANARY).all()
    return dout, out, lse, grads


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 2), (4, 2), (3, 1), (8, 1), (12, 2), (16, 1), (32, 1), (7, 7)])
def test_lengths_and_groups(heads, kv_heads, dim, causal):
    for i, lens in enumerate(LENS):
        _check(*make(lens, heads, kv_heads, dim, 100 * heads + i), causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim,lens", [
    (16, 4, 128, (2048, 333, 1500, 64)), (24, 24, 64, (1537, 900, 4)), (8, 8, 128, (4000,)), (40, 8, 128, (500,) * 9),
    (2, 1, 64, (7, 300) * 40),
])
def test_larger(heads, kv_heads, dim, lens, causal):
    _check(*make(lens, heads, kv_heads, dim, 5), causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_other_rows_hold_does_not_matter(dim, causal):
    lens, lead = (50, 130, 77), 3
    q, k, v, cu = make(lens, 4, 2, dim, 7, lead=lead, tail=9)
    dout, out, lse, want = _check(q, k, v, cu, causal)
    for t, x in ((q, float("nan")), (k, float("inf")), (v, float("nan")), (dout, float("inf")), (out, float("nan"))):
        t[:lead] = x
        t[lead + 50:lead + 180] = x
        t[lead + sum(lens):] = x
    lse[:, :lead] = lse[:, lead + 50:lead + 180] = lse[:, lead + sum(lens):] = float("nan")
    got = [torch.full(t.shape, CANARY, dtype=torch.bfloat16, device="cuda") for t in want]
    hb.packed_backward(dout, q, k, v, out, lse, *got, cu, causal=causal)
    assert hb.packed_status() == 0
    for g, w in zip(got, want):
        for r in (slice(lead, lead + 50), slice(lead + 180, lead + 257)):
            assert torch.equal(g[r], w[r])
        for r in (slice(0, lead), slice(lead + 257, None)):
            assert (g[r] == CANARY).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens", [(2,) * 200, (5, 3, 2, 4) * 40, (20, 10, 33, 128, 127)])
def test_short_sequences_keep_their_precision(lens, dim, causal):
    """Two roundings to bf16 remain, of dS (or P) and of the result.  Each is off by 1.7e-3 of the value in the root mean
    square (up to 2^-8, evenly spread over half a step, over a binade), together 2.4e-3 of the norm; delta taken from the
    rounded output would add as much again and more."""
    q, k, v, cu = make(lens, 4, 2, dim, 8)
    dout, out, lse, grads = _check(q, k, v, cu, causal)
    err, norm = [0.0] * 3, [0.0] * 3
    for a, b, want, _ in _reference(dout, q, k, v, cu, causal, 0.0):
        for i in range(3):
            err[i] += float((grads[i][a:b].double() - want[i]).square().sum())
            norm[i] += float(want[i].square().sum())
    for e, n in zip(err, norm):
        assert math.sqrt(e / n) <= 3e-3, math.sqrt(e / n)


@pytest.mark.parametrize("causal", [True, False])
def test_scales_and_layouts(causal):
    q, k, v, cu = make((300, 20, 170), 6, 2, 64, 9)
    _check(q, k, v, cu, causal, scale=0.3)
    dout, out, lse, want = _check(q, k, v, cu, causal)
    # heads first, and gradients side by side in the layout of the projection
    first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (dout, q, k, v, out)]
    dqkv = torch.full((490, 10, 64), CANARY, dtype=torch.bfloat16, device="cuda")
    got = dqkv[:, :6], dqkv[:, 6:8], dqkv[:, 8:]
    hb.packed_backward(*first, lse, *got, cu, causal=causal)
    assert all(torch.equal(g, w) for g, w in zip(got, want))


@pytest.mark.parametrize("causal", [True, False])
def test_many_short_sequences(causal):
    lens = [int(n) for n in torch.randint(0, 12, (2000,), generator=torch.Generator().manual_seed(1))]
    q, k, v, cu = make(lens, 4, 2, 64, 6, tail=5)
    dout, out, lse = _tensors(q, k, v, cu, causal, 2)
    full = [torch.full(t.shape, CANARY, dtype=torch.bfloat16, device="cuda") for t in (q, k, v)]
    hb.packed_backward(dout, q, k, v, out, lse, *full, cu, causal=causal)
    _check(q, k, v, cu[:60].contiguous(), causal)
    for a in range(0, 2000, 400):
        part = [torch.full_like(t, CANARY) for t in full]
        hb.packed_backward(dout, q, k, v, out, lse, *part, cu[a:a + 401].contiguous(), causal=causal)
        r = slice(int(cu[a]), int(cu[a + 400]))
        assert all(torch.equal(p[r], f[r]) for p, f in zip(part, full))
    assert all((f[int(cu[-1]):] == CANARY).all() for f in full)
    assert hb.packed_status() == 0


def test_gradients_against_differences():
    """Central differences of the forward formula in 64 bits along random directions; the kernel's part of the
    comparison is its own tolerance, 5e-3 of the gradient's norm against a direction of norm one."""
    q, k, v, cu = make((9, 30), 4, 2, 64, 14)
    dout, out, lse, grads = _check(q, k, v, cu, True)

    def loss(q, k, v):
        total = 0.0
        for a, b in ((0, 9), (9, 39)):
            qs, ks, vs = (t[a:b].transpose(0, 1) for t in (q, k, v))
            ks, vs = (t.repeat_interleave(2, 0) for t in (ks, vs))
            s = (qs @ ks.transpose(1, 2) / 8).masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device="cuda").triu(1), -math.inf)
            total = total + (torch.softmax(s, -1) @ vs * dout[a:b].double().transpose(0, 1)).sum()
        return float(total)

    args = [t.double() for t in (q, k, v)]
    g = torch.Generator().manual_seed(15)
    for i, grad in enumerate(grads):
        for _ in range(4):
            d = torch.randn(args[i].shape, generator=g, dtype=torch.float64).cuda()
            d /= d.norm()
            h = 1e-4
            up, down = list(args), list(args)
            up[i], down[i] = args[i] + h * d, args[i] - h * d
            diff = (loss(*up) - loss(*down)) / (2 * h)
            assert abs(diff - float((grad.double() * d).sum())) <= 1e-2 * float(grad.double().norm())


@pytest.mark.parametrize("lens", [(5, 60), (2000, 1000, 200)])
def test_same_bits_again_on_other_streams_and_from_a_graph(lens):
    q, k, v, cu = make(lens, 8, 2, 128, 11)
    dout, out, lse, want = _check(q, k, v, cu, True)
    got = [torch.empty_like(w) for w in want]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        hb.packed_backward(dout, q, k, v, out, lse, *got, cu, stream=side)
        side.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hb.packed_forward(q, k, v, out, cu, lse=lse)
        hb.packed_backward(dout, q, k, v, out, lse, *got, cu)
    n = sum(lens)
    cu.copy_(torch.tensor([0, n // 3, n] if len(lens) == 2 else [0, n // 5, n // 2, n], dtype=torch.int32))
    q.mul_(0.5)
    hb.packed_forward(q, k, v, out, cu, lse=lse)
    hb.packed_backward(dout, q, k, v, out, lse, *want, cu)
    for t in got:
        t.fill_(CANARY)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(g, w) for g, w in zip(got, want))


def test_two_calls_at_once():
    a = []
    for x in (make((700, 300), 4, 4, 64, 20), make((100, 1000, 50), 8, 2, 128, 21)):
        a.append((x, _check(*x, True)))
    streams = [torch.cuda.Stream() for _ in a]
    for _ in range(5):
        got = [[torch.empty_like(w) for w in t[3]] for _, t in a]
        torch.cuda.synchronize()
        for (x, t), o, st in zip(a, got, streams):
            hb.packed_backward(t[0], *x[:3], t[1], t[2], *o, x[3], stream=st)
        torch.cuda.synchronize()
        for (_, t), o in zip(a, got):
            assert all(torch.equal(g, w) for g, w in zip(o, t[3]))
    assert hb.packed_status() == 0


@pytest.mark.parametrize("cu", [(0, 400), (-50, 100, 300), (200, 100, 250), (250, 0), (0, 100, 50, 250)])
def test_bad_lengths_stay_inside(cu):
    q, k, v, good = make((300,), 4, 2, 64, 12)
    dout, out, lse = _tensors(q, k, v, good, True, 3)
    big = [torch.full((500, h, 64), CANARY, dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2)]
    hb.packed_backward(dout, q, k, v, out, lse, *(b[100:400] for b in big), torch.tensor(cu, dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert hb.packed_status() == 0
    for b in big:
        assert (b[:100] == CANARY).all() and (b[400:] == CANARY).all()


def test_refusals():
    q, k, v, cu = make((30,), 4, 2, 64, 13)
    dout, out, lse = _tensors(q, k, v, cu, True, 4)
    g = [torch.empty(t.shape, dtype=torch.bfloat16, device="cuda") for t in (q, k, v)]
    with pytest.raises(ValueError):
        hb.packed_backward(dout, q, k, v, out, None, *g, cu)
    with pytest.raises(ValueError):
        hb.packed_backward(dout, q, k, v, out, lse, g[0], g[1], g[2][:, :1], cu)
    for bad in ((g[0], g[1], g[1]), (q, g[1], g[2]), (g[0], v, g[2]), (dout, g[1], g[2])):
        with pytest.raises(hb.HilbertaError):
            hb.packed_backward(dout, q, k, v, out, lse, *bad, cu)
    with pytest.raises(hb.HilbertaError) as e:
        hb.packed_backward(dout, q, k, v, out, lse, *g, cu, workspace=torch.empty(hb.packed_workspace(30, 4) - 16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == hb.ERR_BUFFER
    hb.packed_backward(dout, q, k, v, out, lse, *g, cu, workspace=torch.empty(hb.packed_workspace(30, 4), dtype=torch.uint8, device="cuda"))
