"""The attention calls take three strides of zero for a contiguous tensor, so the binding hands on none of a row that is broadcast over sequences,
heads and positions.  No GPU."""
import pytest
import torch

from paper_2410_01485_b200 import binding as lg, synth


@pytest.mark.parametrize("which", range(4))
def test_rows_broadcast_over_everything(which):
    p = lg.attn_params(2, 4, 4, 96, 64, 64, synth.MODE_FULL_CAUSAL)
    t = [torch.zeros(2, 4, 96, 64, dtype=torch.bfloat16) for _ in range(4)]
    lg._set_strides(p, *t)
    t[which] = torch.zeros(64, dtype=torch.bfloat16).expand(2, 4, 96, 64)
    assert t[which].stride() == (0, 0, 0, 1)
    with pytest.raises(AssertionError):
        lg._set_strides(p, *t)
    one = torch.zeros(64, dtype=torch.bfloat16).as_strided((1, 1, 1, 64), (0, 0, 0, 1))       # one row is what it says
    lg._set_strides(p, one, one, one, one)
