"""moe_clip_gradients where the norm passes binary32's range."""
import pytest
import torch

pytestmark = pytest.mark.gpu

F, B = torch.float32, torch.bfloat16


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("dtype", [F, B])
def test_a_norm_above_the_range_scales_nothing(dtype, in_place):
    """Finite gradients whose norm is reported as infinity."""
    import paper_2605_11537_amd as moe
    grads = [torch.full((3,), 3e38, device="cuda").to(dtype), torch.randn(5000, device="cuda").to(dtype)]
    kept = [g.clone() for g in grads]
    norm, out = moe.moe_clip_gradients(grads, 1.0, out=grads if in_place else None)
    assert torch.isinf(norm).all() and all(torch.equal(a, b) for a, b in zip(out, kept))

