"""What the binding of the operators around the block refuses by itself, before the library or a device is asked (no GPU needed)."""
import pytest
import torch

from paper_2410_07531_amd import binding as rov


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-50, -1.0, float("nan")])
@pytest.mark.parametrize("given", [False, True])
def test_a_scale_of_zero_does_not_ask_for_two_bytes_an_element(scale, given):
    # the library takes a scale of 0 as "yn in x's type": bf16 values in a buffer of bytes would end behind it
    x, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.ones(64, dtype=torch.bfloat16)
    yn = torch.zeros(4, 64, dtype=torch.uint8) if given else None
    with pytest.raises(ValueError, match="yn_fp8_scale"):
        rov.norm_residual(x, x, w_pre=w, yn=yn, yn_fp8_scale=scale)
