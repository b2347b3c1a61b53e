"""CPU checks of what the binding of a step's calls refuses."""
import pytest
import torch

import paper_2607_21475_amd as ebd
from paper_2607_21475_amd import paged


def _norm(weight):
    """What head_norm makes of weights on the GPU."""
    n = paged.ebd_norm()
    n.eps, n.keep = 1e-6, weight
    n.head_stride = weight.stride(0) if weight.dim() == 2 and weight.shape[0] > 1 else 128 if weight.dim() == 2 else 0
    return n


def test_gradients_of_one_row_of_weights_expanded():
    x = torch.zeros((4, 3, 128), dtype=torch.bfloat16)
    row = torch.ones(128)
    with pytest.raises(ValueError, match="expanded"):
        ebd.norm_rope_backward_params(x, x, x, _norm(row.expand(3, 128)))
    for w in (row, row.repeat(3, 1)):  # (refused for where they are alone)
        with pytest.raises(ValueError, match="on the GPU"):
            ebd.norm_rope_backward_params(x, x, x, _norm(w))
    with pytest.raises(ValueError, match="on the GPU"):
        ebd.norm_rope_params(x, x, _norm(row.expand(3, 128)))
