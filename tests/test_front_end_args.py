"""What the Python entry points of the operators on rows refuse by themselves, before anything reaches the library (no GPU needed)."""
import pytest
import torch

from paper_2412_04747_amd import autograd as A


@pytest.mark.parametrize("out_dtype", [torch.float16, torch.float64, torch.int32, torch.complex64])
def test_residual_norm_writes_fp32_or_bf16(out_dtype):
    with pytest.raises(TypeError, match="out_dtype"):
        A.residual_norm(torch.zeros(3, 8), torch.ones(8), out_dtype=out_dtype)
    with pytest.raises(TypeError, match="fp32 or bf16"):
        A._code(out_dtype)
