"""Calls of a step through the binding on the GPU that the other tests do not make."""
import pytest
import torch

import paged_ref as ref
import step_ref as step

pytestmark = pytest.mark.gpu
BF = torch.bfloat16
EPS = 1e-6


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def test_one_row_of_weights_expanded_over_the_heads():
    """The forward call takes it; its gradient is that of the row, which the gradients' call asks for."""
    import paper_2607_21475_amd as ebd

    g = _gen(3)
    x, dy = ref.spaced((19, 5, 128), g, False), ref.spaced((19, 5, 128), g, False)
    row = 1 + 0.3 * torch.randn(128, generator=g, device="cuda")
    wide = ebd.head_norm(row.expand(5, 128), EPS)
    y = torch.empty_like(x)
    ebd.ebd_norm_rope(ebd.norm_rope_params(x, y, wide), x, y)
    ref.check(y, *step.norm_rope(x, row, EPS, None, None), "y")
    dx = torch.empty_like(x)
    with pytest.raises(ValueError, match="expanded"):
        ebd.norm_rope_backward_params(x, dy, dx, wide)
    p = ebd.norm_rope_backward_params(x, dy, dx, ebd.head_norm(row, EPS))
    dw = torch.full((128,), 7.0, device="cuda")
    ebd.ebd_norm_rope_backward(p, x, dy, dx, dw, ebd.workspace(ebd.ebd_workspace_size(ebd.EBD_WS_NORM_ROPE_BACKWARD, p)))
    (rx, tx), (rw, tw) = step.norm_rope_gradients(x, row, EPS, dy, None, None)
    ref.check(dx, rx, tx, "dx")
    ref.check(dw, rw, tw, "dw")
