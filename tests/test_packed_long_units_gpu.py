"""A unit of work that takes longer than the bounded waits of a block: one key tile that streams the queries of very many heads."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu


def test_a_unit_of_more_than_a_second():
    """65521 heads (a prime: they cannot be shared out) over one key head, 1536 tokens: 786252 blocks a key tile.

    Only three heads have a gradient, so that the sums are those of three heads and sums of zeros, whose roundings are none."""
    T, H, D = 1536, 65521, 64
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    g = torch.Generator(device="cuda").manual_seed(60)
    make = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    # q: windows of one line of numbers, 8 apart: heads share elements, which an input may
    step = 8 * H + D
    q = make(T * step).as_strided((T, H, D), (step, 8, 1))
    k, v = make(T, 1, D), make(T, 1, D)
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    some = [0, 30011, H - 1]
    qs, ds = q[:, some].contiguous(), make(T, 3, D)
    outs, lses = torch.empty_like(qs), torch.empty((3, T), device="cuda")
    hb.packed_forward(qs, k, v, outs, cu, lse=lses, causal=False)
    dout, out = torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda"), torch.zeros((T, H, D), dtype=torch.bfloat16, device="cuda")
    lse = torch.full((H, T), 30.0, device="cuda")
    dout[:, some], out[:, some], lse[some] = ds, outs, lses
    dq, dk, dv = torch.empty_like(dout), torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    hb.packed_backward(dout, q, k, v, out, lse, dq, dk, dv, cu, causal=False)
    end.record()
    assert hb.packed_status() == 0
    print("ms:", start.elapsed_time(end))
    assert start.elapsed_time(end) > 1000   # else this is no test
    want = [torch.empty_like(t) for t in (qs, k, v)]
    hb.packed_backward(ds, qs, k, v, outs, lses, *want, cu, causal=False)
    assert torch.equal(dq[:, some], want[0])
    dq[:, some] = 0
    assert int((dq != 0).sum()) == 0
    # The same products in another order, both results rounded to bf16: 2^-8 each.  Before that 4608 terms, 16 a step, in fp32
    # sums that the tensor cores may truncate: 288 steps of 2^-23 of the running sum, twice, is below 1e-4 of the largest.
    for got, ref in ((dk, want[1]), (dv, want[2])):
        size = float(ref.float().abs().max())
        assert ((got.float() - ref.float()).abs() <= 2.0 ** -7 * ref.float().abs() + 1e-4 * size).all()
    del q, dout, out, lse, dq
    torch.cuda.empty_cache()


def test_more_than_a_second_without_a_unit():
    """65536 sequences, all empty but the last: 396 million units that are not there, one after the other."""
    T, H, D = 65536, 6000, 64
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB of device memory")
    step = 8 * H + D
    line = torch.randn(T * step + 128, generator=torch.Generator(device="cuda").manual_seed(61), device="cuda", dtype=torch.bfloat16)
    q, k, v = (line.as_strided((T, H, D), (step, 8, 1), 64 * i) for i in range(3))
    out = torch.full((T, H, D), 7.0, dtype=torch.bfloat16, device="cuda")
    # one token at the very end: its output is its value
    cu = torch.full((65537,), T - 1, dtype=torch.int32, device="cuda")
    cu[-1] = T
    start, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    hb.packed_forward(q, k, v, out, cu)
    end.record()
    assert hb.packed_status() == 0
    print("ms:", start.elapsed_time(end))
    assert start.elapsed_time(end) > 1000   # else this is no test
    assert torch.equal(out[-1], v[-1])
    assert (out[:-1] == 7.0).all()
    del line, q, k, v, out
    torch.cuda.empty_cache()
