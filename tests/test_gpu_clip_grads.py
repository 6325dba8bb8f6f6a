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


def test_strided_gradients_given_twice():
    from paper_2412_04747_amd import autograd as A
    view = torch.ones(6, 8, device="cuda")[:, ::2]
    p = _param(view)
    for twice in ([p, p], [p, _param(view[:3])]):
        with pytest.raises(RuntimeError, match="share memory"):
            A.clip_grad_norm_(twice, 0.1)
    assert (view == 1.0).all()
    both = torch.full((6, 8), 2.0, device="cuda")        # columns in turn: neither has an element of the other
    norm = A.clip_grad_norm_([_param(both[:, ::2]), _param(both[:, 1::2])], 1.0)
    want = math.sqrt(48 * 4.0)
    assert abs(float(norm) - want) < 1e-6 * want and (both - 2.0 / want).abs().max() < 1e-6


def test_autograd_sees_that_gradients_changed():
    """A graph that saved a gradient must not be walked back over the clipped values."""
    from paper_2412_04747_amd import autograd as A
    p = torch.nn.Parameter(torch.ones(4, device="cuda"))
    p.grad = torch.full((4,), 3.0, device="cuda")
    q = torch.ones(4, device="cuda", requires_grad=True)
    loss = (q * p.grad).sum()
    A.clip_grad_norm_([p], 1.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
