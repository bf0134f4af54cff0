"""Attention over packed sequences against the formula in 64 bits.

Tolerances of `out`, relative to max |v| of the sequence (out is a weighted mean of its rows): weights are rounded to
bf16 before they meet v, off by 2^-9 each (half a step of the value's binade is at most 2^-8 of the value, 2^-9 for the
larger half), which moves a weighted mean by at most 2^-8 max |v|; a quarter of them carry the polynomial's 8e-5
besides.  Scores are fp32 sums of exact products, HD / 16 steps and the adds within one, each off by 2^-23 of the sum of
magnitudes at most: an error e_s that moves weights by 2 e_s.  The result's own rounding is 2^-8 |out|.  lse: e_s, the
weights' 8e-5 at worst, the logarithm's and the result's rounding: 1e-4 + e_s + 2^-23 |lse|."""
import math

import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu

CANARY = 7.0


def make(lens, heads, kv_heads, dim, seed, lead=0, tail=0, gain=1.5, fused=True):
    """q, k, v [total, heads, dim] (slices of one projection if fused) and cu_seqlens; lead / tail: rows outside."""
    g = torch.Generator().manual_seed(seed)
    T = lead + sum(lens) + tail
    cu = torch.tensor([lead] + [lead + sum(lens[:i + 1]) for i in range(len(lens))], dtype=torch.int32).cuda()
    x = (gain * torch.randn((T, heads + 2 * kv_heads, dim), generator=g)).bfloat16().cuda()
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    return q, k, v, cu


def reference(q, k, v, cu, causal, scale=None):
    """Per sequence: its rows, the masked scores and the values in 64 bits, and how far fp32 scores may be off."""
    H, Hk, D = q.shape[1], k.shape[1], q.shape[2]
    scale = D ** -0.5 if scale is None else scale
    bounds = cu.tolist()
    for a, b in zip(bounds, bounds[1:]):
        if b <= a:
            continue
        qs, ks, vs = (t[a:b].double().transpose(0, 1) for t in (q, k, v))
        ks, vs = (t.repeat_interleave(H // Hk, 0) for t in (ks, vs))
        s = qs @ ks.transpose(1, 2) * scale
        e = (D / 16 + 5) * 2.0 ** -23 * float((qs.abs() @ ks.abs().transpose(1, 2)).amax()) * scale
        if causal:
            s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device=q.device).triu(1), -math.inf)
        yield a, b, s, vs, e


def check_forward(q, k, v, cu, causal, scale=0.0, out=None, lse=True):
    T, H, D = q.shape
    out = torch.full((T, H, D), CANARY, dtype=torch.bfloat16, device="cuda") if out is None else out
    ls = torch.full((H, T), CANARY, device="cuda") if lse else None
    hb.packed_forward(q, k, v, out, cu, lse=ls, causal=causal, scale=scale)
    assert hb.packed_status() == 0
    mine = torch.zeros(T, dtype=torch.bool, device="cuda")
    for a, b, s, vs, e in reference(q, k, v, cu, causal, scale or None):
        mine[a:b] = True
        p = torch.softmax(s, -1)
        want = p @ vs
        got = out[a:b].double().transpose(0, 1)
        top = vs.abs().amax((1, 2), keepdim=True)
        assert ((got - want).abs() <= 2.0 ** -8 * (want.abs() + top) + (1e-4 + 2 * e) * top).all(), float((got - want).abs().max())
        rel = float((got - want).norm() / want.norm())
        assert rel <= 5e-3 + 2 * e, rel
        if lse:
            l = torch.logsumexp(s, -1)
            assert ((ls[:, a:b].double() - l).abs() <= 1e-4 + e + 2.0 ** -23 * l.abs()).all()
    assert (out[~mine] == CANARY).all()
    if lse:
        assert (ls[:, ~mine] == CANARY).all()
    return out, ls


LENS = [
    (1,), (2,), (127,), (128,), (129,), (255, 1), (256,), (257,), (1, 1, 1), (0, 5, 0), (640,), (1000, 3, 129, 0, 77, 384),
    tuple(range(1, 40)),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (2, 2), (4, 2), (3, 1), (8, 1), (12, 2), (16, 1), (32, 1), (7, 7)])
def test_lengths_and_groups(heads, kv_heads, dim, causal):
    for i, lens in enumerate(LENS):
        q, k, v, cu = make(lens, heads, kv_heads, dim, 100 * heads + i)
        check_forward(q, k, v, cu, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads,kv_heads,dim,lens", [
    (16, 4, 128, (2048, 333, 1500, 64)), (24, 24, 64, (1537, 900, 4, 2049)), (8, 8, 128, (5000,)), (40, 8, 128, (700,) * 9),
    (2, 1, 64, (7, 300) * 60),
])
def test_larger(heads, kv_heads, dim, lens, causal):
    q, k, v, cu = make(lens, heads, kv_heads, dim, 5)
    check_forward(q, k, v, cu, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
def test_many_short_sequences(dim, causal):
    lens = [int(n) for n in torch.randint(0, 12, (3000,), generator=torch.Generator().manual_seed(1))]
    q, k, v, cu = make(lens, 4, 2, dim, 6, tail=5)
    out, ls = check_forward(q[:0], k[:0], v[:0], cu[:1], causal)
    out = torch.full(q.shape, CANARY, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, q.shape[0]), CANARY, device="cuda")
    hb.packed_forward(q, k, v, out, cu, lse=lse, causal=causal)
    assert hb.packed_status() == 0
    # the first and last hundred sequences against the formula, the others against a call of their own
    check_forward(q, k, v, cu[:101].contiguous(), causal)
    check_forward(q, k, v, cu[-101:].contiguous(), causal)
    for a in range(0, 3000, 500):
        o = torch.full_like(out, CANARY)
        hb.packed_forward(q, k, v, o, cu[a:a + 501].contiguous(), causal=causal)
        r = slice(int(cu[a]), int(cu[a + 500]))
        assert torch.equal(o[r], out[r])
    assert (out[int(cu[-1]):] == CANARY).all()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
def test_what_other_rows_hold_does_not_matter(dim, causal):
    """Rows outside the sequences and a whole neighbouring sequence of NaN and infinities."""
    lens, lead = (50, 130, 77), 3
    q, k, v, cu = make(lens, 4, 2, dim, 7, lead=lead, tail=9)
    out, lse = check_forward(q, k, v, cu, causal)
    for t, x in ((q, float("nan")), (k, float("inf")), (v, float("nan"))):
        t[:lead] = x
        t[lead + 50:lead + 180] = x
        t[lead + sum(lens):] = x
    o, s = torch.full(out.shape, CANARY, dtype=torch.bfloat16, device="cuda"), torch.full_like(lse, CANARY)
    hb.packed_forward(q, k, v, o, cu, lse=s, causal=causal)
    assert hb.packed_status() == 0
    for r in (slice(lead, lead + 50), slice(lead + 180, lead + 257)):
        assert torch.equal(o[r], out[r]) and torch.equal(s[:, r], lse[:, r])
    for r in (slice(0, lead), slice(lead + 257, None)):
        assert (o[r] == CANARY).all() and (s[:, r] == CANARY).all()


@pytest.mark.parametrize("causal", [True, False])
def test_scores_of_all_sizes(causal):
    """Nearly one-hot rows, equal rows, scales given by the caller, and growing scores that move the reference maximum."""
    q, k, v, cu = make((700, 129), 4, 4, 128, 8, gain=6.0)
    check_forward(q, k, v, cu, causal)
    check_forward(q, k, v, cu, causal, scale=0.5)
    check_forward(q * 0, k, v, cu, causal)
    ramp = torch.linspace(0.01, 8.0, q.shape[0], device="cuda")[:, None, None]
    check_forward(q.abs(), (k.abs() * ramp).bfloat16(), v, cu, causal, scale=0.01)
    check_forward(q.abs(), (k.abs() * ramp.flip(0)).bfloat16(), v, cu, causal, scale=0.01)


@pytest.mark.parametrize("causal", [True, False])
def test_layouts(causal):
    """Slices of a projection, separate tensors, heads first, an output inside a wider buffer: the same bits."""
    q, k, v, cu = make((300, 20, 170), 6, 2, 64, 9)
    out, lse = check_forward(q, k, v, cu, causal)
    first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    o, s = check_forward(*first, cu, causal)
    assert torch.equal(o, out) and torch.equal(s, lse)
    wide = torch.full((490, 9, 72), CANARY, dtype=torch.bfloat16, device="cuda")
    o = wide[:, 2:8, 8:72]
    check_forward(q.contiguous(), k.contiguous(), v.contiguous(), cu, causal, out=o, lse=False)
    assert torch.equal(o, out)
    assert (wide[:, :2] == CANARY).all() and (wide[:, 8:] == CANARY).all() and (wide[:, :, :8] == CANARY).all()
    # out in the place of q's neighbours: slices of one buffer
    buf = torch.full((490, 16, 64), CANARY, dtype=torch.bfloat16, device="cuda")
    buf[:, :6], buf[:, 6:8], buf[:, 8:10] = q, k, v
    hb.packed_forward(buf[:, :6], buf[:, 6:8], buf[:, 8:10], buf[:, 10:], cu, causal=causal)
    assert torch.equal(buf[:, 10:], out) and torch.equal(buf[:, :6], q)


def test_offsets_beyond_32_bits():
    """Token strides that take the last rows more than 2^31 elements away."""
    T, stride = 130, 2 ** 24
    q, k, v, cu = make((100, 30), 2, 1, 64, 10)
    big = torch.empty(T * stride + 512, dtype=torch.bfloat16, device="cuda")
    qb, kb, vb, ob = (big.as_strided((T, h, 64), (stride, 64, 1), at) for h, at in ((2, 0), (1, 128), (1, 192), (2, 256)))
    for dst, src in ((qb, q), (kb, k), (vb, v)):
        dst.copy_(src)
    out, _ = check_forward(q, k, v, cu, True)
    hb.packed_forward(qb, kb, vb, ob, cu)
    assert torch.equal(ob, out)


@pytest.mark.parametrize("lens", [(5, 60), (3000, 1000, 200)])
def test_same_bits_again_on_other_streams_and_from_a_graph(lens):
    q, k, v, cu = make(lens, 8, 2, 128, 11)
    out, lse = check_forward(q, k, v, cu, True)
    o, s = torch.empty_like(out), torch.empty_like(lse)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        hb.packed_forward(q, k, v, o, cu, lse=s, stream=side)
        side.synchronize()
        assert torch.equal(o, out) and torch.equal(s, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        hb.packed_forward(q, k, v, o, cu, lse=s)
    # other lengths in the same buffers: they are read on the device
    n = sum(lens)
    cu.copy_(torch.tensor([0, n // 3, n], dtype=torch.int32) if len(lens) == 2 else torch.tensor([0, n // 5, n // 2, n - 1], dtype=torch.int32))
    want, wlse = check_forward(q, k, v, cu, True)
    o.fill_(CANARY)
    s.fill_(CANARY)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(s, wlse)


def test_two_launches_at_once():
    a = [make((700, 300), 4, 4, 64, 20), make((100, 1000, 50), 8, 2, 128, 21)]
    want = [check_forward(*x, True)[0] for x in a]
    streams = [torch.cuda.Stream() for _ in a]
    for _ in range(5):
        got = [torch.empty_like(w) for w in want]
        torch.cuda.synchronize()
        for x, o, st in zip(a, got, streams):
            hb.packed_forward(*x[:3], o, x[3], stream=st)
        torch.cuda.synchronize()
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    assert hb.packed_status() == 0


@pytest.mark.parametrize("cu", [(0, 400), (-50, 100, 300), (200, 100, 250), (0, 2 ** 31 - 1), (300, 300), (250, 0), (0, 100, 50, 250)])
def test_bad_lengths_stay_inside(cu):
    """Offsets that leave the buffer or go back: undefined rows, but only rows of the buffer, and no fault or timeout."""
    q, k, v, _ = make((300,), 4, 2, 64, 12)
    big = torch.full((500, 4, 64), CANARY, dtype=torch.bfloat16, device="cuda")
    hb.packed_forward(q, k, v, big[100:400], torch.tensor(cu, dtype=torch.int32).cuda())
    torch.cuda.synchronize()
    assert hb.packed_status() == 0
    assert (big[:100] == CANARY).all() and (big[400:] == CANARY).all()


def test_refusals():
    q, k, v, cu = make((30,), 4, 2, 64, 13)
    out = torch.empty((30, 4, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        hb.packed_forward(q, k, v, out[:29], cu)
    with pytest.raises(ValueError):
        hb.packed_forward(q, k, v[:, :1], out, cu)
    with pytest.raises(ValueError):
        hb.packed_forward(q, k, v, out, cu.long())
    with pytest.raises(ValueError):
        hb.packed_forward(q, k, v, out, cu.cpu())
    with pytest.raises(ValueError):
        hb.packed_forward(q, k, v, out, cu, lse=torch.empty((30, 4), device="cuda"))
    with pytest.raises(hb.HilbertaError):
        hb.packed_forward(q, k, v, q, cu)
    with pytest.raises(hb.HilbertaError) as e:
        hb.packed_forward(q.float(), k.float(), v.float(), out.float(), cu)
    assert e.value.status == hb.ERR_UNSUPPORTED
    with pytest.raises(hb.HilbertaError):   # 3 key heads do not divide 4
        hb.packed_forward(q, q[:, :3], q[:, :3], out, cu)
