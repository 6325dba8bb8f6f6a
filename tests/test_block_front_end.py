"""What the Python entry points of the junction and of rows in 8 bits refuse by themselves, before anything reaches the library (no GPU needed)."""
import pytest
import torch

from paper_2412_04747_amd import autograd as A
from paper_2412_04747_amd import harness as H

x, w = torch.zeros(6, 8), torch.ones(8)
kinds = torch.zeros(6, dtype=torch.int32)


@pytest.mark.parametrize("kind,word,call", [
    (TypeError, "out_dtype", lambda: A.block_norm(x, x, w, out_dtype=torch.float16)),
    (TypeError, "fp32 or bf16", lambda: A.block_norm(x.half(), x.half(), w)),
    (TypeError, "fp32 or bf16", lambda: A.block_norm(x, x.double(), w)),
    (ValueError, "one shape", lambda: A.block_norm(x, x[:3], w)),
    (ValueError, "one shape", lambda: A.block_norm(torch.zeros(()), torch.zeros(()), w)),
    (ValueError, "one shape", lambda: A.block_norm(torch.zeros(3, 0), torch.zeros(3, 0), w)),
    (TypeError, "w_after", lambda: A.block_norm(x, x, w.bfloat16())),
    (TypeError, "gate", lambda: A.block_norm(x, x, w, w, w.double())),
    (ValueError, "w_before", lambda: A.block_norm(x, x, w, w[:4])),
    (ValueError, "w_after", lambda: A.block_norm(x, x, w.view(1, 8))),
    (ValueError, "gate", lambda: A.block_norm(x, x, w, w, torch.ones(2, 3, 8))),
    (ValueError, "gate", lambda: A.block_norm(x, x, w, w, torch.ones(0, 8))),
    (ValueError, "scale", lambda: A.block_norm(x, x, w, w, w, torch.ones(2, 2))),
    (ValueError, "types", lambda: A.block_norm(x, x, w, w, torch.ones(2, 8), torch.ones(3), kinds)),
    (ValueError, "types", lambda: A.block_norm(x, x, w, w, torch.ones(2, 8))),
    (TypeError, "int32", lambda: A.block_norm(x, x, w, w, torch.ones(2, 8), None, kinds.long())),
    (ValueError, "types", lambda: A.block_norm(x, x, w, w, torch.ones(2, 8), None, kinds[:3])),
    (TypeError, "GPU", lambda: A.block_norm(x, x, w, w, torch.ones(2, 8), torch.ones(2), kinds)),
    (TypeError, "CUDA", lambda: A.pack_rows(x)),
    (TypeError, "int8", lambda: A.unpack_rows(x, x)),
    (TypeError, "GPU", lambda: A.unpack_rows(x.char(), x.byte())),
])
def test_refused(kind, word, call):
    with pytest.raises(kind, match=word):
        call()


def test_rows8_takes_what_it_is_made_for():
    R = H.Rows8.__new__(H.Rows8)
    R.rows, R.width, R._descs = 6, 8, {torch.float32: None, torch.bfloat16: None}
    for bad in (x, x.half(), x[:3], x.t()):
        with pytest.raises(TypeError, match="Rows8"):
            R._desc(bad)


@pytest.mark.parametrize("grad_mode", ["no_grad", "inference_mode", "enabled"])
def test_rows_are_held_only_for_a_backward(grad_mode, monkeypatch):
    """Parameters ask for gradients in evaluation too: whether a graph is recorded decides."""
    asked = {}
    monkeypatch.setattr(A._BlockNorm, "apply", staticmethod(lambda *args: asked.update(block=args[2])))
    monkeypatch.setattr(A._GatedFfn, "apply", staticmethod(lambda *args: asked.update(ffn=args[1])))
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    weights = [torch.nn.Parameter(torch.ones(*shape)) for shape in ((8,), (8, 4), (8, 4), (4, 8))]
    with {"no_grad": torch.no_grad, "inference_mode": torch.inference_mode, "enabled": torch.enable_grad}[grad_mode]():
        A.block_norm(x, x, weights[0], held=True)
        A.gated_ffn(x, *weights[1:], held=True)
        assert asked == dict(block=grad_mode == "enabled", ffn=grad_mode == "enabled")
        A.block_norm(x, x, weights[0])
        A.gated_ffn(x, *weights[1:])
        assert asked == dict(block=False, ffn=False)


def test_buffers_of_the_harness(monkeypatch):
    """What a caller puts in a buffer's place has its type and size: a kernel writes or reads all of it."""
    from paper_2412_04747_amd import binding as B
    monkeypatch.setattr(torch.Tensor, "is_cuda", True)
    R = H.Rows8.__new__(H.Rows8)
    R.rows, R.width = 6, 40
    good = dict(codes=torch.zeros(6, 40, dtype=torch.int8), scales=torch.zeros(6, 2, dtype=torch.uint8))
    L = H.BlockNormLayer.__new__(H.BlockNormLayer)
    L.desc = B.make_block_norm_desc(6, 40, B.RGNN_F32, B.RGNN_BF16, B.RGNN_BF16, 3)
    rows = torch.zeros(6, 40)
    block = dict(a=rows, s=rows.bfloat16(), dOut=rows.bfloat16(), dSum=rows.bfloat16(), types=torch.zeros(6, dtype=torch.int32), w_after=torch.ones(40),
                 w_before=torch.ones(40), gate=torch.ones(3, 40), scale=torch.ones(3))
    for owner, tensors in ((R, good), (L, block)):
        for name, t in tensors.items():
            setattr(owner, name, t)
            assert getattr(owner, name) is t
            for bad in (t[:-1], torch.cat([t, t]), t.double(), t.repeat_interleave(2, -1)[..., ::2], t.long(), None if owner is R else t.half()):
                with pytest.raises(TypeError, match=name):
                    setattr(owner, name, bad)
                assert getattr(owner, name) is t
    monkeypatch.setattr(torch.Tensor, "is_cuda", False)
    with pytest.raises(TypeError, match="codes"):
        R.codes = good["codes"].clone()
    with pytest.raises(TypeError, match="gate"):
        L.gate = block["gate"].clone()
    L.gate = None
    F = H.FfnLayer.__new__(H.FfnLayer)
    F.desc, F.held = B.make_ffn_desc(rows=7, width=64, hidden=10), R
    with pytest.raises(ValueError, match="held"):
        F.bwd_held()
