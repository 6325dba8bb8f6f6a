"""`clip_grad_norm_` of gradients that torch allows and the kernel does not see: views, shared memory, versions."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def _param(grad):
    p = torch.nn.Parameter(torch.zeros(grad.shape, device="cuda", dtype=grad.dtype))
    p.grad = grad
    return p


def test_an_expanded_gradient_is_refused_before_anything_is_scaled():
    from paper_2412_04747_amd import autograd as A
    first = _param(torch.full((5, 3), 2.0, device="cuda"))
    for bad in (torch.ones(1, 4, device="cuda").expand(6, 4), torch.ones((), device="cuda").expand(7),
                torch.ones(8, device="cuda").as_strided((3, 4), (2, 1))):
        with pytest.raises(RuntimeError, match="share memory"):
            A.clip_grad_norm_([first, _param(bad)], 0.1)
        assert (first.grad == 2.0).all()
    # strides that step over each other are fine, and so is an empty one
    apart = torch.full((4, 6), 3.0, device="cuda")[:, ::2].t()
    norm = A.clip_grad_norm_([first, _param(apart), _param(torch.ones(0, 4, device="cuda"))], 1.0)
    want = math.sqrt(15 * 4.0 + 12 * 9.0)
    assert abs(float(norm) - want) < 1e-6 * want and (apart - 3.0 / want).abs().max() < 1e-6
