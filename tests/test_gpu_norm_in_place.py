"""Residual norm written over its inputs: the same bits as into other memory, at rows of every kind (several to a wavefront, a wavefront's, a
workgroup's; odd widths in unaligned vectors), types and accumulation."""
import pytest

from test_gpu_row_norm import _inputs, _layer

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,width", [(1003, 64), (77, 33), (301, 349), (40, 1024), (37, 2048), (9, 4099), (21, 8192)])
@pytest.mark.parametrize("types", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "f32"), ("bf16", "f32", "f32")])
def test_over_its_inputs(rows, width, types):
    import torch
    print(f"norm case rows={rows} width={width} types {types}", flush=True)
    x, total, out = types
    d = _inputs(rows, width, x, total, out, True, 9)
    L, M = (_layer(d, rows, width, x, total, out, True) for _ in range(2))
    L.fwd(); L.bwd()
    # sum over residual; out over x, where it is of x's type
    M.sum = M.residual
    if out == x:
        M.out = M.x
    M.fwd()
    assert torch.equal(M.sum, L.sum) and torch.equal(M.out, L.out)
    # the residual's gradient over dSum, x's over dOut, or where they are one buffer, that over dSum
    if M.dX is not None and out == x:
        M.dX = M.dOut
    M.dResidual = M.dSum
    M.bwd()
    assert torch.equal(M.dResidual, L.dResidual) and torch.equal(M.dWeight, L.dWeight)
    if M.dX is not None:
        assert torch.equal(M.dX, L.dX)


@pytest.mark.parametrize("width", [64, 349, 4099])
def test_sum_over_x(width):
    import torch
    rows = 50
    d = _inputs(rows, width, "f32", "f32", "bf16", True, 3)
    L, M = (_layer(d, rows, width, "f32", "f32", "bf16", True) for _ in range(2))
    L.fwd()
    M.sum = M.x
    M.fwd()
    assert torch.equal(M.sum, L.sum) and torch.equal(M.out, L.out)
