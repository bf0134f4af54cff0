"""The operators around the sparse attention, as cases that can be timed and compared.

A case is one call of one operator, as a training step or a serving loop makes it:

  norm, norm_grad      layer norm over the last axis, affine or modulated by one scale and shift per sample as
                       diffusion transformers use it, and its gradients (input, scale, shift)
  rotary, rotary_grad  rotary positions on q or k: interleaved and half layouts, part of the head, one position
                       axis or several, frequencies scaled for long contexts, with or without the entry gather
                       into the plan's physical order; and the gradient, with or without the exit gather
  packed, packed_grad  attention over whole sequences of different lengths packed one after the other (prompts
                       of a text encoder, images of several sizes), causal or not, heads in groups; and its
                       gradients

With `own` false, run() computes the operators from elementary torch operations in 32 bits (angles in 64); with
`own` true it calls the library.  exact() is the definition in 64 bits, written apart from both.
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_SIZE = {"bf16": 2, "fp32": 4}
_DEV = "cuda"
# Limits of the drawn cases: elements of one norm or rotary tensor, padded scores of the plain packed attention.
_MOST_ELEMENTS, _MOST_SCORES = 5.0e7, 1.0e9


def _norm(name, op, batch, rows, cols, dtype, wdtype, modulated):
    return dict(name=name, op=op, batch=batch, rows=rows, cols=cols, dtype=dtype, wdtype=wdtype, modulated=modulated)


def _rotary(name, op, batch, heads, S, dim, pairs, dtype, interleaved=False, scaling=1.0, far=0, packed=False, grid=0,
            text=0):
    """grid > 0: image tokens on a grid x grid plan behind `text` text tokens, three position axes, with the gather."""
    return dict(name=name, op=op, batch=batch, heads=heads, S=S, dim=dim, pairs=pairs, dtype=dtype,
                interleaved=interleaved, scaling=scaling, far=far, packed=packed, grid=grid, text=text)


def _packed(name, op, lens, heads, kv_heads, dim, causal, tail=0):
    """lens: sequence lengths; tail: rows of the buffers behind the last sequence."""
    return dict(name=name, op=op, lens=",".join(str(n) for n in lens), heads=heads, kv_heads=kv_heads, dim=dim,
                causal=causal, tail=tail)


def listed():
    return [
        # serving: the norm in front of a layer for a handful of single tokens
        _norm("norm_tokens", "norm", 1, 4, 1536, "bf16", "bf16", False),
        # 2048^2 image, two samples: the modulated norm in front of a block's attention
        _norm("norm_modulated_2048", "norm", 2, 16896, 1536, "bf16", "bf16", True),
        # training at 1024^2, eight samples, weights kept in fp32
        _norm("norm_grad_1024", "norm_grad", 8, 4608, 1152, "bf16", "fp32", False),
        # fp32 training of a model of odd width, three samples of odd length, modulated
        _norm("norm_grad_odd_fp32", "norm_grad", 3, 1777, 777, "fp32", "fp32", True),
        # serving: one new token for each of sixteen sequences far into a scaled context
        _rotary("rotary_tokens", "rotary", 16, 32, 1, 128, 64, "bf16", scaling=8.0, far=900000),
        # 2048^2 image: q of one layer on its way into the physical order, positions on three axes
        _rotary("rotary_entry_2048", "rotary", 1, 24, 16896, 128, 64, "bf16", interleaved=True, grid=128, text=512),
        # fp32 training on packed tokens: the gradient where only part of an odd-sized head is rotated
        _rotary("rotary_grad_packed_fp32", "rotary_grad", 1, 9, 5001, 80, 24, "fp32", packed=True),
        # a text encoder's batch: prompts of a few tokens up to the usual limit
        _packed("packed_prompts", "packed", (77, 9, 1, 20, 64, 33, 12, 77, 5, 48), 12, 12, 64, True, tail=51),
        # a large text encoder on long documents, four query heads to a key head
        _packed("packed_documents", "packed", (4096, 3333, 2900, 1911), 32, 8, 128, True),
        # images of three sizes with their prompts, every token sees its whole sequence
        _packed("packed_images", "packed", (4608, 2816, 1541), 24, 24, 128, False),
        # training on documents, four query heads to a key head
        _packed("packed_grad_documents", "packed_grad", (2048, 1500, 4096, 333), 16, 4, 128, True),
        # training on short prompts, three query heads to a key head
        _packed("packed_grad_prompts", "packed_grad", (77, 300, 1, 120, 511, 64, 77, 250), 12, 4, 64, True, tail=8),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(("norm", "norm_grad", "rotary", "rotary_grad", "packed", "packed_grad"))
    if op.startswith("norm"):
        cols = _log_int(rng, 64, 8192)
        if rng.random() < 0.7:
            cols = (cols + 7) // 8 * 8
        batch = rng.choice((1, 1, 2, 3, 8))
        rows = _log_int(rng, 1, max(1, min(40000, int(_MOST_ELEMENTS / cols / batch))))
        c = _norm("", op, batch, rows, cols, rng.choice(("bf16", "bf16", "fp32")), rng.choice(("same", "fp32")), rng.random() < 0.5)
        if c["wdtype"] == "same":
            c["wdtype"] = c["dtype"]
    elif op.startswith("rotary"):
        dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 128, 192, 256))
        pairs = dim // 2 if rng.random() < 0.6 else rng.randint(1, dim // 2)
        heads = rng.choice((1, 2, 3, 8, 12, 24, 32))
        inter, dtype = rng.random() < 0.5, rng.choice(("bf16", "bf16", "fp32"))
        if rng.random() < 0.3:
            grid, text = rng.choice((16, 24, 32, 50, 64, 100, 128)), rng.choice((0, 3, 77, 512))
            batch = 1 if grid > 64 else rng.choice((1, 2))
            if dtype == "fp32":
                heads = min(heads, 12)
            c = _rotary("", op, batch, heads, grid * grid + text, dim, max(pairs, 3), dtype, inter, grid=grid, text=text)
        else:
            batch = rng.choice((1, 2, 5, 16))
            S = _log_int(rng, 1, max(1, min(32768, int(_MOST_ELEMENTS / dim / heads / batch))))
            c = _rotary("", op, batch, heads, S, dim, pairs, dtype, inter, rng.choice((1.0, 1.0, 4.0, 16.0)),
                        rng.choice((0, 0, 4000, 2000000)), rng.random() < 0.5)
    else:
        kv_heads, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 1, 2, 3, 4, 6, 8))
        n, longest = _log_int(rng, 1, 40), _log_int(rng, 1, 8192)
        most = _MOST_SCORES / 2 if op == "packed_grad" else _MOST_SCORES
        while n > 1 and n * kv_heads * group * longest ** 2 > most:
            n = max(1, n // 2)
        while kv_heads * group * longest ** 2 > most:
            longest = longest * 2 // 3
        lens = [longest] + [rng.randint(0, longest) if rng.random() < 0.5 else _log_int(rng, 1, longest) for _ in range(n - 1)]
        rng.shuffle(lens)
        c = _packed("", op, lens, kv_heads * group, kv_heads, rng.choice((64, 128)), rng.random() < 0.7, rng.choice((0, 0, 1, 100)))
    del c["name"]
    return c


# ---- inputs ----------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=_DEV).manual_seed(seed)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device=_DEV)


def _frequencies(pairs, scaling):
    """base^(-j / pairs) in 64 bits; scaled: wavelengths beyond the trained context slowed by `scaling`, those
    well inside it kept, a linear ramp between (1 to 32 turns over 4096 tokens)."""
    f = 10000.0 ** (-torch.arange(pairs, dtype=torch.float64) / pairs)
    if scaling == 1.0:
        return f, 1.0
    ramp = ((4096 * f / (2 * math.pi) - 1.0) / 31.0).clamp(0, 1)
    return f * (ramp + (1 - ramp) / scaling), 1.0 + 0.1 * math.log(scaling)


def _lens(case):
    return [int(n) for n in case["lens"].split(",")]


def prepare(case, seed):
    g = _generator(seed)
    s = dict(case)
    dt = _DTYPES[case["dtype"]] if "dtype" in case else torch.bfloat16
    if case["op"].startswith("norm"):
        B, R, C = case["batch"], case["rows"], case["cols"]
        # activations with an offset and rows of different sizes, as a residual stream has them
        x = (_randn(g, B, R, C) * (0.5 + 2 * torch.rand((B, R, 1), generator=g, device=_DEV)) + 0.3 * _randn(g, 1, 1, C)).to(dt)
        wshape, around = ((B, C), 0.0) if case["modulated"] else ((C,), 1.0)
        s.update(x=x, eps=1e-6, weight=(around + 0.2 * _randn(g, *wshape)).to(_DTYPES[case["wdtype"]]),
                 bias=(0.2 * _randn(g, *wshape)).to(_DTYPES[case["wdtype"]]))
        if case["op"] == "norm_grad":
            xf = x.double()
            mean = xf.mean(-1)
            rstd = (xf.var(-1, correction=0) + s["eps"]).rsqrt()
            s.update(dy=_randn(g, B, R, C).to(dt), mean=mean.float(), rstd=rstd.float(), dx=torch.empty_like(x),
                     dweight=torch.empty_like(s["weight"]), dbias=torch.empty_like(s["bias"]))
        else:
            s.update(y=torch.empty_like(x), mean=torch.empty((B, R), device=_DEV), rstd=torch.empty((B, R), device=_DEV))
    elif case["op"].startswith("rotary"):
        B, H, S, D = case["batch"], case["heads"], case["S"], case["dim"]
        if case["packed"]:   # [B, S, heads, D] as a projection leaves it
            x = _randn(g, B, S, H, D).to(dt).transpose(1, 2)
            out = torch.empty((B, S, H, D), dtype=dt, device=_DEV).transpose(1, 2)
        else:
            x, out = _randn(g, B, H, S, D).to(dt), torch.empty((B, H, S, D), dtype=dt, device=_DEV)
        s.update(x=x, out=out, axis=None, plan=None)
        if case["grid"]:
            from paper_2509_26538_b200 import binding as hb
            G, nt = case["grid"], case["text"]
            padded = 1 << (G - 1).bit_length()
            s["plan"] = hb.Plan(G, G, padded * padded // 4, padded * padded // 8, 4, nt)
            s["phys2orig"] = torch.from_numpy(s["plan"].export(hb.EXPORT_PHYS2ORIG)).to(_DEV)
            cell = torch.arange(G * G, device=_DEV)
            # text tokens count on the first axis, image tokens are rows and columns on the other two
            pos = torch.zeros((S, 3), dtype=torch.int32, device=_DEV)
            pos[:nt, 0] = torch.arange(nt, device=_DEV, dtype=torch.int32)
            pos[nt:, 1] = (cell // G).int()
            pos[nt:, 2] = (cell % G).int()
            per = [case["pairs"] // 8, (case["pairs"] - case["pairs"] // 8) // 2]
            per.append(case["pairs"] - sum(per))
            s["positions"] = pos
            s["axis"] = torch.repeat_interleave(torch.arange(3), torch.tensor(per)).to(torch.int32)
            s["inv_freq"], s["factor"] = torch.cat([_frequencies(p, 1.0)[0] for p in per]), 1.0
        else:
            start = torch.randint(0, case["far"] + 1, (B, 1), generator=g, device=_DEV)
            s["positions"] = (start + torch.arange(S, device=_DEV)).int()
            s["inv_freq"], s["factor"] = _frequencies(case["pairs"], case["scaling"])
    else:
        lens, Hq, Hk, D = _lens(case), case["heads"], case["kv_heads"], case["dim"]
        T = sum(lens) + case["tail"]
        cu = torch.tensor([0] + lens).cumsum(0).to(device=_DEV, dtype=torch.int32)
        # one projection's output: q, k and v of a token side by side
        qkv = (1.5 * _randn(g, T, Hq + 2 * Hk, D)).to(dt)
        q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hk], qkv[:, Hq + Hk:]
        s.update(q=q, k=k, v=v, cu=cu, longest=max(lens), out=torch.zeros((T, Hq, D), dtype=dt, device=_DEV),
                 lse=torch.zeros((Hq, T), device=_DEV))
        if case["op"] == "packed_grad":
            s["out"], s["lse"] = _packed_forward(s)
            s["dout"] = _randn(g, T, Hq, D).to(dt)
            s["dq"], s["dk"], s["dv"] = (torch.zeros((T, h, D), dtype=dt, device=_DEV) for h in (Hq, Hk, Hk))
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------

def _wide(w):
    """Weights per sample stand against [batch, rows, cols]."""
    return w.float().unsqueeze(1) if w.dim() == 2 else w.float()


def _norm_forward(s):
    x = s["x"].float()
    mean = x.mean(-1, keepdim=True)
    d = x - mean
    rstd = ((d * d).mean(-1, keepdim=True) + s["eps"]).rsqrt()
    w = _wide(s["weight"]) + (1.0 if s["modulated"] else 0.0)
    y = d * rstd * w + _wide(s["bias"])
    return y.to(s["x"].dtype), mean.squeeze(-1), rstd.squeeze(-1)


def _norm_backward(s):
    dy, rstd = s["dy"].float(), s["rstd"].unsqueeze(-1)
    n = (s["x"].float() - s["mean"].unsqueeze(-1)) * rstd
    gy = dy * (_wide(s["weight"]) + (1.0 if s["modulated"] else 0.0))
    dx = rstd * (gy - gy.mean(-1, keepdim=True) - n * (gy * n).mean(-1, keepdim=True))
    over = 1 if s["modulated"] else (0, 1)
    return dx.to(s["x"].dtype), (dy * n).sum(over).to(s["weight"].dtype), dy.sum(over).to(s["bias"].dtype)


def _rotary_plain(s, sign):
    x, pairs = s["x"], s["pairs"]
    if s["plan"] is not None:
        if sign > 0:
            x = x[:, :, s["phys2orig"].long()]
        else:
            x = torch.empty_like(x).index_copy_(2, s["phys2orig"].long(), x)
    pos, freq = s["positions"], s["inv_freq"].to(_DEV)
    if s["axis"] is not None:
        angle = pos[:, s["axis"].to(_DEV).long()].double() * freq
        if sign > 0:
            angle = angle[s["phys2orig"].long()]
    else:
        angle = (pos.unsqueeze(-1).double() * freq).unsqueeze(1)
    cos, sin = (s["factor"] * angle.cos()).float(), (sign * s["factor"] * angle.sin()).float()
    head, rest = x[..., :2 * pairs].float(), x[..., 2 * pairs:]
    a, b = (head[..., 0::2], head[..., 1::2]) if s["interleaved"] else (head[..., :pairs], head[..., pairs:])
    a, b = a * cos - b * sin, a * sin + b * cos
    head = torch.stack((a, b), -1).flatten(-2) if s["interleaved"] else torch.cat((a, b), -1)
    return torch.cat((head.to(x.dtype), rest), -1)


def _padded(s):
    """Row of the buffers for each place of a [sequences, longest] block, which places hold a token, and for each row
    its sequence and place."""
    cu, L = s["cu"].long(), s["longest"]
    lens, at = cu[1:] - cu[:-1], torch.arange(L, device=_DEV)
    T = s["q"].shape[0]
    row = (cu[:-1, None] + at).clamp(max=T - 1)
    t = torch.arange(T, device=_DEV)
    seq = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=len(lens) - 1)
    return row, at < lens[:, None], seq, (t - cu[seq]).clamp(0, L - 1), t < cu[-1]


def _heads_first(t, row, heads):
    t = t[row].permute(0, 2, 1, 3).float()   # [sequences, heads, longest, dim]
    return t if t.shape[1] == heads else t.repeat_interleave(heads // t.shape[1], 1)


def _masked_scores(s, qp, kp, held):
    L = s["longest"]
    seen = held[:, None, None, :]
    if s["causal"]:
        seen = seen & torch.ones((L, L), dtype=torch.bool, device=_DEV).tril()
    return torch.matmul(qp, kp.transpose(-1, -2)).mul_(s["dim"] ** -0.5).masked_fill_(~seen, -math.inf)


def _rows(s, t, seq, place, live, behind):
    """[sequences, heads, longest, dim] back to rows; rows behind the last sequence keep what they hold."""
    return torch.where(live[:, None, None], t.permute(0, 2, 1, 3)[seq, place].to(behind.dtype), behind)


def _packed_forward(s):
    row, held, seq, place, live = _padded(s)
    H = s["heads"]
    score = _masked_scores(s, _heads_first(s["q"], row, H), _heads_first(s["k"], row, H), held)
    score.masked_fill_(~held[:, None, :, None], 0.0)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p, _heads_first(s["v"], row, H)) / total
    lse = (top + total.log()).squeeze(-1).permute(0, 2, 1)[seq, place]
    lse = torch.where(live[:, None], lse, s["lse"].t()).t().contiguous()
    return _rows(s, out, seq, place, live, s["out"]), lse


def _packed_backward(s):
    row, held, seq, place, live = _padded(s)
    H, scale = s["heads"], s["dim"] ** -0.5
    qp, kp, vp, gp = (_heads_first(s[n], row, H) for n in ("q", "k", "v", "dout"))
    gp = gp * held[:, None, :, None]
    p = _masked_scores(s, qp, kp, held).sub_(s["lse"].t()[row].permute(0, 2, 1).unsqueeze(-1)).exp_()
    p.masked_fill_(~held[:, None, :, None], 0.0)
    dv = torch.matmul(p.transpose(-1, -2), gp)
    ds = torch.matmul(gp, vp.transpose(-1, -2))
    ds = ds.sub_((p * ds).sum(-1, keepdim=True)).mul_(p)
    dq = torch.matmul(ds, kp).mul_(scale)
    dk = torch.matmul(ds.transpose(-1, -2), qp).mul_(scale)
    shared = lambda t: t.unflatten(1, (s["kv_heads"], -1)).sum(2)  # noqa: E731
    return (_rows(s, dq, seq, place, live, s["dq"]), _rows(s, shared(dk), seq, place, live, s["dk"]),
            _rows(s, shared(dv), seq, place, live, s["dv"]))


def run(state):
    s, op = state, state["op"]
    if own:
        from paper_2509_26538_b200 import binding as hb
        if op == "norm":
            return hb.layer_norm(s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"], eps=s["eps"],
                                 unit_offset=s["modulated"])
        if op == "norm_grad":
            return hb.layer_norm_backward(s["dy"], s["x"], s["weight"], s["mean"], s["rstd"], s["dx"], s["dweight"],
                                          s["dbias"], unit_offset=s["modulated"])
        if op == "rotary" or op == "rotary_grad":
            f = hb.rotary if op == "rotary" else hb.rotary_backward
            return f(s["x"], s["out"], s["inv_freq"], s["positions"], axis=s["axis"], interleaved=s["interleaved"],
                     factor=s["factor"], plan=s["plan"])
        if op == "packed":
            return hb.packed_forward(s["q"], s["k"], s["v"], s["out"], s["cu"], lse=s["lse"], causal=s["causal"])
        return hb.packed_backward(s["dout"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dq"], s["dk"], s["dv"],
                                  s["cu"], causal=s["causal"])
    if op == "norm":
        return _norm_forward(s)
    if op == "norm_grad":
        return _norm_backward(s)
    if op == "rotary" or op == "rotary_grad":
        return _rotary_plain(s, 1.0 if op == "rotary" else -1.0)
    return _packed_forward(s) if op == "packed" else _packed_backward(s)


def _pairs_seen(case):
    return sum(n * (n + 1) // 2 if case["causal"] else n * n for n in _lens(case))


def work(case):
    if case["op"].startswith("norm"):
        n, rows = case["batch"] * case["rows"] * case["cols"], case["batch"] * case["rows"]
        w = 2 * _SIZE[case["wdtype"]] * case["cols"] * (case["batch"] if case["modulated"] else 1)
        grad = case["op"] == "norm_grad"
        return {"bytes": n * _SIZE[case["dtype"]] * (3 if grad else 2) + 8 * rows + (2 * w if grad else w), "flops": n * (14 if grad else 8)}
    if case["op"].startswith("rotary"):
        rows = case["batch"] * case["heads"] * case["S"]
        index = 4 * case["S"] * (4 if case["grid"] else case["batch"])
        return {"bytes": 2 * rows * case["dim"] * _SIZE[case["dtype"]] + index, "flops": 6 * rows * case["pairs"]}
    T, Hq, Hk, D = sum(_lens(case)), case["heads"], case["kv_heads"], case["dim"]
    if case["op"] == "packed":
        return {"bytes": T * (2 * D * (2 * Hq + 2 * Hk) + 4 * Hq), "flops": 4 * D * Hq * _pairs_seen(case)}
    return {"bytes": T * (2 * D * (4 * Hq + 4 * Hk) + 4 * Hq), "flops": 10 * D * Hq * _pairs_seen(case)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------

def _exact_norm(s):
    x = s["x"].double()
    B, R, C = x.shape
    w, b = (s[n].double().reshape(-1, 1, C) for n in ("weight", "bias"))
    if s["modulated"]:
        w = w + 1
    mean, var = x.mean(2), x.var(2, correction=0)
    n = (x - mean[..., None]) / torch.sqrt(var + s["eps"])[..., None]
    if s["op"] == "norm":
        return n * w + b, mean, 1 / torch.sqrt(var + s["eps"])
    dy = s["dy"].double()
    gy = dy * w
    dx = (gy - gy.sum(2, keepdim=True) / C - n * ((gy * n).sum(2, keepdim=True) / C)) / torch.sqrt(var + s["eps"])[..., None]
    dw, db = torch.einsum("brc,brc->bc", dy, n), dy.sum(1)
    if not s["modulated"]:
        dw, db = dw.sum(0), db.sum(0)
    return dx, dw, db


def _exact_rotary(s):
    x = s["x"].double()
    B, H, S, D = x.shape
    back = s["op"] == "rotary_grad"
    pos = s["positions"].double()
    if s["axis"] is None:
        angle = torch.einsum("bs,p->bsp", pos, s["inv_freq"].to(_DEV))
    else:
        angle = torch.stack([pos[:, int(a)] * float(f) for a, f in zip(s["axis"], s["inv_freq"])], -1).expand(B, S, -1)
    if s["plan"] is not None:
        if back:   # row p of the gradient belongs to token phys2orig[p]
            x = x[:, :, torch.argsort(s["phys2orig"].long())]
        else:
            x, angle = x[:, :, s["phys2orig"].long()], angle[:, s["phys2orig"].long()]
    turn = torch.polar(torch.full_like(angle, s["factor"]), -angle if back else angle)[:, None]
    out, P = x.clone(), s["pairs"]
    first, second = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if s["interleaved"] else (slice(0, P), slice(P, 2 * P))
    z = torch.complex(x[..., first], x[..., second]) * turn
    out[..., first], out[..., second] = z.real, z.imag
    return out


def _exact_packed(s):
    Hq, Hk, D = s["heads"], s["kv_heads"], s["dim"]
    names = ("out", "lse") if s["op"] == "packed" else ("dq", "dk", "dv")
    got = {n: s[n].double() for n in names}
    at = 0
    for n in _lens(s):
        r = slice(at, at + n)
        at += n
        for h in range(Hq if n else 0):
            j = h // (Hq // Hk)
            q, k, v = s["q"][r, h].double(), s["k"][r, j].double(), s["v"][r, j].double()
            score = q @ k.t() / math.sqrt(D)
            if s["causal"]:
                score = score.masked_fill(torch.ones((n, n), dtype=torch.bool, device=_DEV).triu(1), -math.inf)
            p = torch.softmax(score, -1)
            if s["op"] == "packed":
                got["out"][r, h], got["lse"][h, r] = p @ v, torch.logsumexp(score, -1)
                continue
            g = s["dout"][r, h].double()
            dp = g @ v.t()
            ds = p * (dp - (p * dp).sum(-1, keepdim=True)) / math.sqrt(D)
            got["dq"][r, h] = ds @ k
            got["dk"][r, j] += ds.t() @ q
            got["dv"][r, j] += p.t() @ g
    return tuple(got[n] for n in names)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("norm"):
        return _exact_norm(s)
    return _exact_rotary(s) if case["op"].startswith("rotary") else _exact_packed(s)
