"""Feed-forward block at sizes where the choice of kernels turns, and where the weights are laid out: tails of rows and hidden values, both
activations, guard zones, rows that stay alone.  Bounds as in `test_gpu_ffn`."""
import pytest

from test_gpu_ffn import _check, _inputs, _layer, expected

pytestmark = pytest.mark.gpu


# width 32 with its chunks divided among four, two and one group of wavefronts; the least and the most rows of either side of a limit
SIZES = [(3001, 32, 130, "bf16"), (3001, 32, 130, "f32"), (9001, 32, 200, "bf16"), (9001, 32, 97, "f32"), (17001, 32, 129, "bf16"), (17001, 32, 300, "f32"),
         (33, 128, 64, "bf16"), (33, 128, 64, "f32"), (700, 128, 40, "f32"), (2, 128, 33, "bf16"), (5, 32, 96, "f32"), (65, 64, 64, "bf16"), (64, 64, 96, "bf16"),
         (495, 32, 128, "bf16"), (496, 32, 128, "bf16"), (6145, 128, 65, "f32"), (3585, 64, 33, "bf16"), (8193, 32, 40, "bf16"), (12289, 32, 257, "f32")]


@pytest.mark.parametrize("rows,width,hidden,dtype", SIZES)
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_against_the_definition(rows, width, hidden, dtype, act):
    import torch
    print(f"ffn case rows={rows} width={width} hidden={hidden} {dtype} {act}", flush=True)
    p = _inputs(rows, width, hidden, dtype, act, 5)
    L = _layer(p, act)
    L.fwd(); L.bwd()
    torch.cuda.synchronize()
    want = expected(p, act, dtype)
    for k, v in (("out", L.out), *L.grads().items()):
        _check(v, want[k], k)


# many rows with relu at every width, the fp32 backward among them
@pytest.mark.parametrize("rows,width,hidden,dtype", [(40001, 32, 70, "f32"), (40001, 32, 70, "bf16"), (9001, 64, 100, "f32"), (9001, 128, 65, "f32"), (20003, 128, 97, "bf16")])
def test_many_rows_relu(rows, width, hidden, dtype):
    import torch
    print(f"ffn case rows={rows} width={width} hidden={hidden} {dtype} relu", flush=True)
    p = _inputs(rows, width, hidden, dtype, "relu", 7)
    L = _layer(p, "relu")
    L.fwd(); L.bwd()
    torch.cuda.synchronize()
    want = expected(p, "relu", dtype)
    for k, v in (("out", L.out), *L.grads().items()):
        _check(v, want[k], k)


@pytest.mark.parametrize("rows,width,hidden,dtype", [(3001, 64, 100, "bf16"), (9001, 64, 100, "bf16"), (20003, 64, 100, "bf16"), (8200, 64, 65, "f32"), (12001, 64, 90, "f32"),
                                                     (9001, 128, 65, "f32"), (20003, 128, 97, "bf16"), (33001, 32, 97, "f32"), (3001, 32, 130, "bf16"), (9001, 32, 130, "f32")])
def test_laid_out_weights_repeatable_bounded_and_alone(rows, width, hidden, dtype):
    """The same bits twice; nothing written behind the last row or the workspace; a row with NaN touches no other row."""
    import torch
    from paper_2412_04747_amd import binding as B
    print(f"ffn case rows={rows} width={width} hidden={hidden} {dtype}", flush=True)
    L = _layer(_inputs(rows, width, hidden, dtype, "silu", 31), "silu")
    L.fwd(); L.bwd()
    first = [t.clone() for t in (L.out, *L.grads().values())]
    big = torch.full((2, rows + 200, width), 7.0, device="cuda", dtype=L.out.dtype)
    f, b = B.rgnn_ffn_workspace_bytes(L.desc)
    ws = torch.full((max(f, b) + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    L.out, L.dX, L.ws = big[0, :rows], big[1, :rows], ws
    L.fwd()
    assert (ws[f:] == 0xA5).all()
    L.bwd()
    assert (ws[max(f, b):] == 0xA5).all() and (big[:, rows:] == 7.0).all()
    for x, y in zip(first, (L.out, *L.grads().values())):
        assert torch.equal(x, y)
    bad = [0, rows // 2, rows - 1]
    L.X[bad[0], 0], L.X[bad[1], 3], L.X[bad[2], width - 1] = float("inf"), float("nan"), float("-inf")
    L.fwd(); L.bwd()
    good = torch.ones(rows, dtype=torch.bool, device="cuda")
    good[bad] = False
    assert torch.equal(L.out[good], first[0][good]) and torch.equal(L.dX[good], first[1][good])
    assert not L.out[bad].isfinite().any()
