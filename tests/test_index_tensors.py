"""Labels and positions are read one behind the other: a view with strides is refused.  No GPU."""
import pytest
import torch

import paper_2407_20761_amd as ob


def test_positions_kept_token_by_token():
    x, desc = torch.zeros(4, 64, dtype=torch.bfloat16), ob.make_rotary_axes_desc([0, 1] * 16, 64)
    pos = torch.zeros((4, 2), dtype=torch.int32).t()
    with pytest.raises(ValueError, match="contiguous"):
        ob.ob_rotary_axes(desc, x, 64, x, 64, 4, 1, pos)
    with pytest.raises(ValueError, match="contiguous"):
        ob.BlockAttn(rotary=desc, pos=pos)
    ob.BlockAttn(rotary=desc, pos=pos.contiguous())


def test_labels_with_strides():
    x, labels, f = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(8, dtype=torch.int32)[::2], torch.zeros(4)
    desc = ob.make_lm_loss_desc(64, 4)
    with pytest.raises(ValueError, match="contiguous"):
        ob.ob_lm_loss_fwd(desc, x, x, 4, None, labels, f, f, x, x)
    with pytest.raises(ValueError, match="contiguous"):
        ob.ob_lm_loss_bwd(desc, 0, x, x, 4, None, labels, f, f, x, x, x, x)
