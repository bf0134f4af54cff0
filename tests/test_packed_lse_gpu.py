"""lse of the packed attention at the accuracy that its polynomial's degree was chosen for.

lse = ln(sum p) + the reference.  A score is an fp32 sum of exact products, off by e at most (see test_packed_gpu.py), and so is
what it adds to lse.  Three quarters of the weights come from the exponential unit, off by 2^-22, a quarter from the polynomial of degree
4, off by 2.7e-6 in the worst place; either works on x = score log2 e - reference, rounded to fp32 once in the product with the scale
and once in the sum: 2^-24 (|x| + 2 |reference|) each.  Sums of positive terms in fp32 chains of 16, then one a block:
2^-24 (20 + blocks) relative.  The logarithm and the last two roundings: 3 * 2^-24 |lse| and 2^-22."""
import math

import pytest
import torch

from paper_2509_26538_b200 import binding as hb
from test_packed_gpu import make, reference

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("lens,gain", [((1, 2, 3, 64, 77), 1.5), ((128, 129, 700), 1.5), ((4096,), 1.5), ((900, 1300), 0.3), ((1000,), 4.0)])
def test_lse_is_as_good_as_degree_four(lens, gain, dim, causal):
    q, k, v, cu = make(lens, 4, 2, dim, 50, gain=gain)
    out, lse = torch.empty_like(q), torch.empty((4, q.shape[0]), device="cuda")
    hb.packed_forward(q, k, v, out, cu, lse=lse, causal=causal)
    for a, b, s, _, e in reference(q, k, v, cu, causal):
        want = torch.logsumexp(s, -1)
        err = (lse[:, a:b].double() - want).abs()
        top = s.masked_fill(s == -math.inf, 0).abs().amax(-1)
        bound = 2.7e-6 + 2.0 ** -22 + e + 4 * U * top + U * (20 + (b - a) / 128) + 3 * U * want.abs() + 2.0 ** -22
        assert (err <= bound).all(), float((err / bound).max())
    assert hb.packed_status() == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("step", range(1, 48, 3))
def test_every_part_of_the_polynomial(step, dim):
    """All keys but the first score -step / 32, exactly: a quarter of the weights are one value of the polynomial."""
    n = 640
    q, k = (torch.zeros((n, 1, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q[:, 0, 0] = 1.0
    k[1:, 0, 0] = -step / 32   # at most six bits
    out, lse = torch.empty_like(q), torch.empty((1, n), device="cuda")
    cu = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    hb.packed_forward(q, k, torch.ones_like(k), out, cu, lse=lse, causal=False, scale=1.0)
    s = k[:, 0, 0].double()
    want = float(torch.logsumexp(s, 0))
    fma = (torch.arange(n, device="cuda") // 2) % 4 == 3
    share = float(s.exp()[fma].sum() / s.exp().sum())
    bound = 2.7e-6 * share + 2.0 ** -22 + 4 * U * step / 32 + U * (20 + n / 128) + 3 * U * want + 2.0 ** -22
    assert float((lse.double() - want).abs().max()) <= bound, float((lse.double() - want).abs().max()) / bound
    assert hb.packed_status() == 0
