"""Elements behind the rotated part are copied bit for bit, NaN payloads among them."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("dim,pairs", [(128, 64), (128, 33), (128, 40), (64, 1), (64, 30), (80, 24), (80, 39), (66, 5), (256, 101)])
def test_the_rest_keeps_its_bits(dim, pairs, interleaved, dtype):
    g = torch.Generator().manual_seed(dim + pairs)
    bits, whole = (torch.int16, 16) if dtype == torch.bfloat16 else (torch.int32, 32)
    # every bit pattern may occur: quiet and signalling NaN, infinities, subnormals, negative zeros
    x = torch.randint(-2 ** (whole - 1), 2 ** (whole - 1), (2, 3, 50, dim), generator=g).to(bits)
    x[..., ::7] = 0x7f81 if whole == 16 else 0x7f800001
    x[..., 1::9] = -1
    x = x.cuda()
    freq, _ = hb.rotary_frequencies(pairs)
    for fn in (hb.rotary, hb.rotary_backward):
        out = torch.zeros_like(x)
        fn(x.view(dtype), out.view(dtype), freq, interleaved=interleaved)
        assert torch.equal(out[..., 2 * pairs:], x[..., 2 * pairs:])
        same = x.clone()
        fn(same.view(dtype), same.view(dtype), freq, interleaved=interleaved)
        assert torch.equal(same[..., 2 * pairs:], x[..., 2 * pairs:])
