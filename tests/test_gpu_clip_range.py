"""Clipping by a coefficient below fp32's normal range: of a norm near fp32's largest value, or past it.  Bounds as in `test_gpu_grad_clip`; values
below 2^-126 are held to multiples of 2^-149 (bf16: 2^-133)."""
import math

import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("values,max_norm", [([3e38, 3e38], 1.0), ([3.3e38] * 1000 + [1e25, -7e31], 1e-3), ([1e36, 2e36, 3e30], 1e-3), ([1e38], 1e-6),
                                             ([2e38, 1e3], 0.5)])
def test_small_coefficients(values, max_norm, bf16):
    import torch
    from paper_2412_04747_amd.harness import GradClip
    print(f"clip case of {len(values)} large values, max_norm {max_norm} bf16={bf16}", flush=True)
    g = [torch.tensor(values, device="cuda").to(torch.bfloat16 if bf16 else torch.float32), torch.full((4097,), 1e33, device="cuda")]
    before = [t.double() for t in g]
    norm = math.sqrt(sum(float(t.pow(2).sum()) for t in before))
    L = GradClip(g)
    L.clip(g, max_norm)
    got = float(L.norm)
    assert abs(got - norm) <= norm * 1.01 * U if norm < 3.4e38 else got == math.inf
    c = max_norm / (norm + 1e-6)
    for b, a in zip(before, g):
        half = a.dtype == torch.bfloat16
        tol = b.abs() * c * ((2.0 ** -8 if half else 0.0) + 2.1 * U) + (2.0 ** -134 if half else 0.0) + 2.0 ** -148
        assert ((a.double() - b * c).abs() <= tol).all()
