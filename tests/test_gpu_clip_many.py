"""Clipping of thousands of tensors: more pieces than the workgroups of the second pass add by themselves.  Bounds as in `test_gpu_grad_clip`."""
import math

import pytest

from test_gpu_grad_clip import _check

pytestmark = pytest.mark.gpu


def _tensors(count, seed):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.randn(4 * count, generator=g, device="cuda")
    return [flat[4 * i:4 * i + 1 + i % 4] for i in range(count)]


@pytest.mark.parametrize("count", [4095, 4096, 4097, 8193, 20011])
def test_against_the_definition(count):
    import torch
    from paper_2412_04747_amd import binding as B
    from paper_2412_04747_amd.harness import GradClip
    print(f"clip case of {count} tensors", flush=True)
    grads = _tensors(count, count)
    whole = torch.cat(grads)
    want = float(whole.double().norm())
    L = GradClip(grads)
    n = B.rgnn_clip_workspace_bytes([t.numel() for t in grads])
    L.ws = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    L.clip(grads, 0.25 * want)
    _check([whole], [torch.cat(grads)], L.norm, 0.25 * want)
    assert (L.ws[n:] == 0xA5).all()
    first = float(L.norm)
    alone = torch.zeros((), device="cuda")               # the norm without clipping
    B.rgnn_clip_grad_norm([whole], None, [whole.numel()], [B.RGNN_F32], 0.0, alone, L.ws)
    assert abs(float(alone) - want) <= want * 1.01 * 2.0 ** -24
    again = _tensors(count, count)
    B.rgnn_clip_grad_norm(again, None, L.sizes, L.dtypes, 0.0, alone, L.ws)
    assert float(alone) == first
    L.clip(again, math.inf)                              # the same bits again, and nothing scaled
    assert float(L.norm) == first and torch.equal(torch.cat(again), whole)


def test_work_grows_with_the_number_of_tensors():
    """A launch takes up to 128 tensors: its time must not grow with the number of all tensors."""
    import torch
    from paper_2412_04747_amd import binding as B
    from paper_2412_04747_amd.harness import GradClip
    each = {}
    for count in (2048, 98304):
        print(f"clip case of {count} tensors", flush=True)
        grads = _tensors(count, 1)
        L = GradClip(grads)
        L.clip(grads, 1e-3)
        torch.cuda.synchronize()
        B.rgnn_profile_start()
        for _ in range(3):
            L.clip(grads, 1e-3)
        launches, ms = B.rgnn_profile_stop()["grad_scale"]
        each[count] = ms / launches
    print(f"  {each}", flush=True)
    assert each[98304] < 2 * each[2048]
