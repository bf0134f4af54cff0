"""What the binding of the block's operators takes and refuses before the library is asked.  No device is needed."""
import pytest
import torch

from paper_2509_26538_b200 import binding as hb


def test_one_row_of_weights_has_any_stride():
    """A single sample's scale and shift as slices of tensors of different widths."""
    x = torch.zeros((1, 3, 8))
    scale, shift = torch.zeros((1, 16))[:, 8:], torch.zeros((1, 24))[:, 8:16]
    assert scale.stride() != shift.stride()
    per, _, code = hb._norm_weights(x, scale, shift)
    assert (per, code) == (0, hb.FP32)
    assert hb._norm_weights(x, torch.zeros((1, 8)), shift)[0] == 0
    one = torch.zeros((2, 3, 1))   # one column: the last axis may have any stride too
    assert hb._norm_weights(one, torch.zeros((2, 4))[:, :1], torch.zeros((2, 4, 2))[:, :1, 0].as_strided((2, 1), (4, 2)))[:2] == (3, 4)
    for a, b in ((torch.zeros((2, 8)), torch.zeros((2, 16))[:, 8:]), (torch.zeros(8), torch.zeros(16)[::2]),
                 (torch.zeros((1, 8)), torch.zeros(8)), (torch.zeros((1, 8)), torch.zeros((1, 8)).bfloat16())):
        with pytest.raises(ValueError):
            hb._norm_weights(x if a.dim() == 1 or a.shape[0] == 1 else torch.zeros((2, 3, 8)), a, b)


def test_a_workspace_is_one_run_of_bytes():
    """Every other byte of a buffer has the right count, but the library would write the bytes between them too."""
    holes = torch.zeros(1 << 16, dtype=torch.uint8)[::2]
    x, st = torch.zeros((4, 8)), torch.zeros(4)
    with pytest.raises(ValueError, match="workspace"):
        hb.layer_norm_backward(x, x, None, st, st, x.clone(), torch.zeros(8), None, workspace=holes)
    q, lse, cu = torch.zeros((4, 1, 64)).bfloat16(), torch.zeros((1, 4)), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="workspace"):
        hb.packed_backward(q, q, q, q, q, lse, q.clone(), q.clone(), q.clone(), cu, workspace=holes)
