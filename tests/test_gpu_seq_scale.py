"""Scales that 32 bits round to 0 are refused: 0 stands for the default scale there."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [1e-46, 1e-60, 0.0, -1.0, float("nan")])
def test_scale_that_is_no_positive_float(scale):
    import torch
    assert torch.cuda.is_available(), "GPU tests need a visible MI355X"
    from paper_2110_14007_amd import tod
    q = torch.randn(3, 2, 64, device="cuda").half()
    starts = torch.tensor([0, 3], dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError):
        tod.tod_attn_prompt(q, q, q, starts, scale=scale)
    # the smallest that there is: every key has the same weight
    out = tod.tod_attn_prompt(q, q, q, starts, causal=False, scale=1e-45)
    want = q.double().mean(0).expand(3, 2, 64)
    assert float((out.double() - want).abs().max()) <= 2.0 ** -10 * float(q.abs().max())
