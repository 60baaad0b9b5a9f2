"""Types that the gradient of the experts' products takes and refuses (no GPU needed: nothing is launched)."""
import pytest
import torch


def test_the_weights_gradient_has_a_type_the_kernels_write():
    from paper_2401_13920_b200 import experts as X
    offsets = torch.tensor([0, 2, 4, 4], dtype=torch.int32)
    dy, x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(4, 16, dtype=torch.bfloat16), torch.zeros(3, 8, 16)
    for bad in (torch.float16, torch.float64):
        with pytest.raises(TypeError, match="dw_dtype"):
            X.expert_linear_grad(dy, x, w.to(bad), offsets, want_dx=False)
        with pytest.raises(TypeError, match="dw_dtype"):
            X.expert_linear_grad(dy, x, w, offsets, want_dx=False, dw_dtype=bad)
    for good in (torch.float32, torch.bfloat16):                     # host memory is what is refused then
        with pytest.raises(ValueError, match="dy"):
            X.expert_linear_grad(dy, x, w.to(good), offsets, want_dx=False)
