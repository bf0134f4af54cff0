"""The operators in a row, as a transformer block uses them, forward and backward, against autograd in 64 bits.

Tolerance: in bf16 every tensor that one operator hands to the next is rounded, off by 1.7e-3 of its norm in the root
mean square; there are a dozen of them between the block's input and its gradient, and the softmax passes an error of the
scores (of size one or two here) on to its weights unchanged.  Twelve such errors add up to 6e-3 of the norm; with a
factor of three for those that are not independent, 2e-2.  In fp32 (the sparse attention's fp32 kernels) the same chain is
held to 1e-4: 2^-24 a rounding, and up to 1e-5 from the attention."""
import math

import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu


def _rel(a, b):
    a, b = a.detach().double(), b.detach().double()
    return float((a - b).norm() / b.norm())


def _randn(g, *shape):
    return torch.randn(shape, generator=g, dtype=torch.float64).cuda()


def _norm64(x, scale, shift):
    n = (x - x.mean(-1, keepdim=True)) / (x.var(-1, correction=0, keepdim=True) + 1e-6).sqrt()
    return n * (1 + scale[:, None]) + shift[:, None]


def _turn64(x, angle, interleaved):
    """x [..., S, D], angle [S, P] or [B, 1, S, P]."""
    P = angle.shape[-1]
    a, b = (x[..., 0:2 * P:2], x[..., 1:2 * P:2]) if interleaved else (x[..., :P], x[..., P:2 * P])
    c, s = angle.cos(), angle.sin()
    u, v = a * c - b * s, a * s + b * c
    head = torch.stack((u, v), -1).flatten(-2) if interleaved else torch.cat((u, v), -1)
    return torch.cat((head, x[..., 2 * P:]), -1)


@pytest.mark.parametrize("dtype,tol", [(torch.bfloat16, 2e-2), (torch.float32, 1e-4)])
def test_image_block_through_the_plan(dtype, tol):
    """norm, projection, rotary positions on three axes with the entry gather, sparse attention with the v gather beside it,
    and all gradients back to the input and the modulation."""
    H, W, text, B, heads, D = 16, 16, 20, 2, 3, 64
    C = heads * D
    plan = hb.Plan(H, W, 64, 16, 2, text)
    S = plan.S
    g = torch.Generator().manual_seed(1)
    x64, scale64, shift64 = _randn(g, B, S, C), 0.2 * _randn(g, B, C), 0.2 * _randn(g, B, C)
    w64, dout64 = _randn(g, C, 3 * C) / math.sqrt(C), _randn(g, B, heads, S, D)
    x, scale, shift, w, dout = (t.to(dtype) for t in (x64, scale64, shift64, w64, dout64))
    pos = torch.zeros((S, 3), dtype=torch.int32)
    pos[:text, 0] = torch.arange(text)
    pos[text:, 1], pos[text:, 2] = torch.arange(H * W) // W, torch.arange(H * W) % W
    axis = torch.tensor([0] * 4 + [1] * 14 + [2] * 14, dtype=torch.int32)
    freq = torch.cat([hb.rotary_frequencies(n)[0] for n in (4, 14, 14)])
    try:
        # ---- the library
        n, mean, rstd = torch.empty_like(x), torch.empty((B, S), device="cuda"), torch.empty((B, S), device="cuda")
        hb.layer_norm(x, scale, shift, n, mean, rstd, unit_offset=True)
        qkv = (n.reshape(-1, C).double() @ w.double()).to(dtype).reshape(B, S, 3, heads, D)
        q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
        qp, kp, vp, out = (torch.empty((B, heads, S, D), dtype=dtype, device="cuda") for _ in range(4))
        dpos = pos.cuda()
        hb.rotary(q, qp, freq, dpos, axis=axis, interleaved=True, plan=plan)
        hb.rotary(k, kp, freq, dpos, axis=axis, interleaved=True, plan=plan)
        plan.permute(v.contiguous(), vp)
        plan.bind_like(qp)
        lse = torch.empty((B, heads, S), device="cuda")
        plan.forward_lse(qp, kp, vp, out, lse)
        y = torch.empty_like(out)
        plan.unpermute(out, y)
        dop = torch.empty_like(out)
        plan.permute(dout, dop)
        dqp, dkp, dvp = (torch.empty_like(out) for _ in range(3))
        plan.backward(dop, qp, kp, vp, out, lse, dqp, dkp, dvp)
        dqkv = torch.empty((B, S, 3, heads, D), dtype=dtype, device="cuda")
        hb.rotary_backward(dqp, dqkv[:, :, 0].transpose(1, 2), freq, dpos, axis=axis, interleaved=True, plan=plan)
        hb.rotary_backward(dkp, dqkv[:, :, 1].transpose(1, 2), freq, dpos, axis=axis, interleaved=True, plan=plan)
        dv = torch.empty_like(dvp)
        plan.unpermute(dvp, dv)
        dqkv[:, :, 2].transpose(1, 2).copy_(dv)
        dn = (dqkv.reshape(-1, 3 * C).double() @ w.double().t()).to(dtype).reshape(B, S, C)
        dx, dscale, dshift = torch.empty_like(x), torch.empty_like(scale), torch.empty_like(shift)
        hb.layer_norm_backward(dn, x, scale, mean, rstd, dx, dscale, dshift, unit_offset=True)
        assert plan.status() == 0
        # ---- 64 bits, in the original token order: the mask by classes
        p2o = torch.from_numpy(plan.export(hb.EXPORT_PHYS2ORIG)).long().cuda()
        windows = plan.export(hb.EXPORT_WINDOWS)
        P = text + int(plan.export(hb.EXPORT_INFO)[6])
        group = torch.full((S,), -1, dtype=torch.long)
        for i, (_, s0, l0, s1, l1) in enumerate(windows.tolist()):
            group[s0:s0 + l0] = i
            group[s1:s1 + l1] = i
        prefix = torch.arange(S) < P
        allowed = (prefix[:, None] | prefix[None] | (group[:, None] == group[None])).cuda()
        mask = torch.empty_like(allowed)
        mask[p2o[:, None], p2o[None]] = allowed
        leaves = [t.double().requires_grad_() for t in (x, scale, shift)]
        rq, rk, rv = (_norm64(*leaves) @ w.double()).reshape(B, S, 3, heads, D).permute(2, 0, 3, 1, 4)
        angle = pos[:, axis.long()].double().cuda() * freq.cuda()
        s = _turn64(rq, angle, True) @ _turn64(rk, angle, True).transpose(-1, -2) / math.sqrt(D)
        ry = torch.softmax(s.masked_fill(~mask, -math.inf), -1) @ rv
        grads = torch.autograd.grad((ry * dout.double()).sum(), leaves)
        assert _rel(y, ry) <= tol
        for got, want in zip((dx, dscale, dshift), grads):
            assert _rel(got, want) <= tol, _rel(got, want)
    finally:
        plan.destroy()


@pytest.mark.parametrize("heads,kv_heads,D,pairs,interleaved", [(4, 2, 64, 32, False), (6, 2, 128, 40, True)])
def test_text_block_on_packed_prompts(heads, kv_heads, D, pairs, interleaved):
    """norm, projection, rotary positions that start again in every prompt (q and k in place in one call), causal attention
    over the packed prompts, and all gradients back to the input and the norm's weights.  Two such blocks' worth of calls
    behind each other on a stream of its own, the second replayed from a graph."""
    lens, C, dtype, tol = (77, 1, 200, 33, 128), 256, torch.bfloat16, 2e-2
    T, N = sum(lens), heads + 2 * kv_heads
    g = torch.Generator().manual_seed(2)
    cu = torch.tensor([0] + list(lens)).cumsum(0).int().cuda()
    pos = torch.cat([torch.arange(n) for n in lens]).int().cuda()
    freq, factor = hb.rotary_frequencies(pairs, scaling=hb.ROTARY_BANDS, scale=4.0, context=64.0)
    x, weight, bias = _randn(g, T, C).to(dtype), (1 + 0.2 * _randn(g, C)).float(), (0.2 * _randn(g, C)).float()
    w, dout = (_randn(g, C, N * D) / math.sqrt(C)).to(dtype), _randn(g, T, heads, D).to(dtype)
    n, mean, rstd = torch.empty_like(x), torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    qkv, dqkv = (torch.empty((T, N, D), dtype=dtype, device="cuda") for _ in range(2))
    out, lse = torch.empty((T, heads, D), dtype=dtype, device="cuda"), torch.empty((heads, T), device="cuda")
    dn, dx, dweight, dbias = torch.empty_like(x), torch.empty_like(x), torch.empty_like(weight), torch.empty_like(bias)
    parts = lambda t: (t[:, :heads], t[:, heads:heads + kv_heads], t[:, heads + kv_heads:])  # noqa: E731

    def block():
        hb.layer_norm(x, weight, bias, n, mean, rstd)
        torch.mm(n, w, out=qkv.view(T, N * D))
        turned = qkv[:, :heads + kv_heads].unsqueeze(0).transpose(1, 2)
        hb.rotary(turned, turned, freq, pos, interleaved=interleaved, factor=factor)
        hb.packed_forward(*parts(qkv), out, cu, lse=lse)
        hb.packed_backward(dout, *parts(qkv), out, lse, *parts(dqkv), cu)
        turned = dqkv[:, :heads + kv_heads].unsqueeze(0).transpose(1, 2)
        hb.rotary_backward(turned, turned, freq, pos, interleaved=interleaved, factor=factor)
        torch.mm(dqkv.view(T, N * D), w.t(), out=dn)
        hb.layer_norm_backward(dn, x, weight, mean, rstd, dx, dweight, dbias)

    def check():
        leaves = [t.double().requires_grad_() for t in (x, weight, bias)]
        nn = (leaves[0] - leaves[0].mean(-1, keepdim=True)) / (leaves[0].var(-1, correction=0, keepdim=True) + 1e-6).sqrt()
        rq, rk, rv = (t.transpose(0, 1) for t in parts(((nn * leaves[1] + leaves[2]) @ w.double()).reshape(T, N, D)))
        angle = pos.double()[:, None] * freq.cuda()
        grow = torch.cat((torch.full((2 * pairs,), factor), torch.ones(D - 2 * pairs))).double().cuda()
        rq, rk = _turn64(rq, angle, interleaved) * grow, _turn64(rk, angle, interleaved) * grow
        seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens)).cuda()
        mask = (seq[:, None] == seq[None]) & torch.ones((T, T), dtype=torch.bool, device="cuda").tril()
        rk, rv = (t.repeat_interleave(heads // kv_heads, 0) for t in (rk, rv))
        s = (rq @ rk.transpose(1, 2) / math.sqrt(D)).masked_fill(~mask, -math.inf)
        ry = (torch.softmax(s, -1) @ rv).transpose(0, 1)
        grads = torch.autograd.grad((ry * dout.double()).sum(), leaves)
        assert hb.packed_status() == 0
        assert _rel(out, ry) <= tol
        for got, want in zip((dx, dweight, dbias), grads):
            assert _rel(got, want) <= tol, _rel(got, want)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        block()
        block()
    side.synchronize()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        block()
    x.copy_(_randn(g, T, C).to(dtype))
    dout.copy_(_randn(g, T, heads, D).to(dtype))
    for t in (out, dx, dweight, dbias):
        t.fill_(float("nan"))
    graph.replay()
    torch.cuda.synchronize()
    check()
