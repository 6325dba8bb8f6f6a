"""What the Python entry points of the operators on rows refuse by themselves, before anything reaches the library (no GPU needed)."""
import pytest
import torch

from paper_2412_04747_amd import autograd as A
from paper_2412_04747_amd import binding as B
from paper_2412_04747_amd import harness as H


@pytest.mark.parametrize("out_dtype", [torch.float16, torch.float64, torch.int32, torch.complex64])
def test_residual_norm_writes_fp32_or_bf16(out_dtype):
    with pytest.raises(TypeError, match="out_dtype"):
        A.residual_norm(torch.zeros(3, 8), torch.ones(8), out_dtype=out_dtype)
    with pytest.raises(TypeError, match="fp32 or bf16"):
        A._code(out_dtype)


@pytest.mark.parametrize("like", [torch.zeros(8, dtype=torch.float16), torch.zeros(8, dtype=torch.float64), torch.zeros(8), torch.zeros(1).expand(8)])
def test_grad_clip_is_made_for_dense_gpu_tensors(like):
    with pytest.raises(TypeError, match="GradClip"):
        H.GradClip([like])


def test_grad_clip_compares_what_it_is_given():
    """(Tensors on the CPU, without a launch: the checks of `clip` alone.)"""
    L = H.GradClip.__new__(H.GradClip)
    L._numel, L._types, L._devices, L._layouts = [6, 4], [torch.float32, torch.bfloat16], [-1, -1], None
    a, b = torch.zeros(2, 3), torch.zeros(4, dtype=torch.bfloat16)
    L._check([a, b])
    for bad in ([a], [a, b, b], [b, a], [a, torch.zeros(4)], [torch.zeros(5), b], [torch.zeros(2, 4), b], [torch.zeros(3, 2).t(), b],
                [torch.zeros(1).expand(6), b], [torch.zeros(12)[::2], b]):
        with pytest.raises(ValueError, match="GradClip"):
            L._check(bad)
    L._layouts = [((2, 3), (1, 2)), ((4,), (1,))]
    L._check([torch.zeros(3, 2).t(), b])
    for bad in (a, torch.zeros(6)):
        with pytest.raises(ValueError, match="layout"):
            L._check([bad, b])


def test_clip_tables_of_one_length():
    """Raw addresses, never read: the lists' lengths are compared first."""
    at = [1 << 28, 1 << 29]
    for grads, clipped, sizes, dtypes in ((at, None, [4], [0, 0]), (at, at, [4, 4], [0]), (at, at[:1], [4, 4], [0, 0]), (at[:1], None, [4, 4], [0, 0]),
                                          (at, at, *B.clip_tables([4], [0]))):
        with pytest.raises(ValueError, match="tensors"):
            B.rgnn_clip_grad_norm(grads, clipped, sizes, dtypes, 1.0, 1 << 30, 1 << 31)


def test_stream_of_a_torch_without_its_internal_call(monkeypatch):
    class Stream:
        cuda_stream = 1234

    monkeypatch.setattr(torch.cuda, "current_stream", lambda device: Stream if device == 3 else None)
    assert H._raw_stream(object())(3) == 1234
    assert H._raw_stream(type("C", (), {"_cuda_getCurrentRawStream": staticmethod(lambda device: device + 1)}))(3) == 4
