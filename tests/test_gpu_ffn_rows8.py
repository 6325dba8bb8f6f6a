"""The feed-forward block's backward from rows held in 8 bits.

A held value is exact in fp32 and in bfloat16, and its second and third planes, which the call does not form, are zeros: products with them add nothing.  So
the gradients are the bits of the call on the unpacked rows; and both are within the bounds of the block's own tests of the definition in 64 bits."""
import pytest

from test_gpu_ffn import _check, _inputs, expected

pytestmark = pytest.mark.gpu

CASES = [(1, 32, 1), (1, 128, 512), (2, 64, 33), (5, 128, 70), (31, 64, 31), (33, 32, 32), (64, 32, 300), (65, 64, 100), (129, 64, 86), (300, 128, 341), (1000, 32, 86), (1000, 128, 128),
         (4099, 64, 256), (9003, 128, 65), (12001, 64, 90), (33001, 32, 97)]


def _held(p, act, flags=0, spread=0.0):
    """The layer with its rows in 8 bits, and p with the values that they stand for."""
    import torch
    from paper_2412_04747_amd.harness import FfnLayer, Rows8
    rows, d = p["X"].shape
    f, t = p["Wg"].shape[1], p["dOut"].dtype
    L = FfnLayer(rows, d, f, "bf16" if t == torch.bfloat16 else "f32", act, flags=flags)
    L.held = Rows8(rows, d)
    x = p["X"].float()
    if spread:
        x = x * torch.exp(spread * torch.randn(rows, d // 32, 1, generator=torch.Generator().manual_seed(1))).expand(rows, d // 32, 32).reshape(rows, d)
    L.held.pack(x.cuda())
    values = torch.empty(rows, d, dtype=t, device="cuda")
    L.held.unpack(values)
    p = dict(p, X=values.cpu())
    for k, v in p.items():
        setattr(L, k, v.cuda())
    return L, p


@pytest.mark.parametrize("rows,width,hidden", CASES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_bits_of_the_unpacked_rows(rows, width, hidden, dtype, act):
    import torch
    print(f"ffn held case rows={rows} width={width} hidden={hidden} {dtype} {act}", flush=True)
    L, p = _held(_inputs(rows, width, hidden, dtype, act, rows + width + hidden), act, spread=1.0 if act == "silu" else 0.0)
    L.bwd_held()
    got = {k: v.clone() for k, v in L.grads().items()}
    L.bwd()
    torch.cuda.synchronize()
    for k, v in L.grads().items():
        assert torch.equal(got[k], v), k


@pytest.mark.parametrize("rows,width,hidden", [(1, 64, 5), (300, 128, 341), (1000, 32, 86), (9003, 128, 65), (12001, 64, 90)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_against_the_definition(rows, width, hidden, dtype):
    import torch
    print(f"ffn held case rows={rows} width={width} hidden={hidden} {dtype}, 64 bits", flush=True)
    L, p = _held(_inputs(rows, width, hidden, dtype, "silu", 5), "silu")
    L.bwd_held()
    torch.cuda.synchronize()
    want = expected(p, "silu", dtype)
    for k, v in L.grads().items():
        _check(v, want[k], k)


@pytest.mark.parametrize("rows,width,hidden,dtype", [(700, 64, 50, "f32"), (700, 128, 50, "bf16"), (20001, 64, 40, "f32")])
def test_wanted_gradients_alone_and_added_to(rows, width, hidden, dtype):
    import torch
    from paper_2412_04747_amd import binding as B
    L, p = _held(_inputs(rows, width, hidden, dtype, "silu", 6), "silu")
    L.bwd_held()
    want = {k: v.clone() for k, v in L.grads().items()}
    w = (L.Wg, L.Wu, L.Wd, L.dOut)
    L.dX.fill_(9.0)
    B.rgnn_ffn_bwd_rows8(L.desc, L.held.tensors(), *w, L.dX, None, None, None, L.ws)
    torch.cuda.synchronize()
    assert torch.equal(L.dX, want["dX"])
    for k in ("dWg", "dWu", "dWd"):
        getattr(L, k).fill_(9.0)
    B.rgnn_ffn_bwd_rows8(L.desc, L.held.tensors(), *w, None, L.dWg, L.dWu, L.dWd, L.ws)
    torch.cuda.synchronize()
    for k in ("dWg", "dWu", "dWd"):
        assert torch.equal(getattr(L, k), want[k]), k
    M, _ = _held(_inputs(rows, width, hidden, dtype, "silu", 6), "silu", flags=B.RGNN_FLAG_ACCUMULATE)
    N, _ = _held(_inputs(rows, width, hidden, dtype, "silu", 6), "silu", flags=B.RGNN_FLAG_ACCUMULATE)
    for q in (M, N):
        for k, v in q.grads().items():
            v.copy_(want[k])
    M.bwd_held()
    N.bwd()
    torch.cuda.synchronize()
    for k, v in M.grads().items():
        assert torch.equal(v, N.grads()[k]), k


def test_a_bad_row_stays_alone():
    import torch
    p = _inputs(400, 64, 60, "f32", "silu", 7)
    L, _ = _held(p, "silu")
    L.bwd_held()
    torch.cuda.synchronize()
    want = L.dX.clone()
    p["X"][9, 40] = float("inf")
    M, _ = _held(p, "silu")
    M.bwd_held()
    torch.cuda.synchronize()
    keep = torch.arange(400, device="cuda") != 9
    assert torch.equal(M.dX[keep], want[keep]) and torch.isnan(M.dX[9]).all()


def test_no_rows():
    import torch
    L, _ = _held(_inputs(0, 64, 60, "f32", "silu", 7), "silu")
    for t in (L.dWg, L.dWu, L.dWd):
        t.fill_(4.0)
    L.bwd_held()
    torch.cuda.synchronize()
    assert not (L.dWg.any() or L.dWu.any() or L.dWd.any())


def test_captured_and_replayed():
    """Packing, forward and the backward from the packed rows in a graph, replayed over changing rows with eager calls between."""
    import torch
    p = _inputs(600, 64, 90, "f32", "silu", 8)
    E, _ = _held(p, "silu")
    L, _ = _held(p, "silu")

    def step(q):
        q.held.pack(q.X)
        q.fwd()
        q.bwd_held()

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step(L)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(L)
    for turn in range(3):
        x = torch.randn(600, 64, generator=torch.Generator().manual_seed(turn)).cuda()
        for q in (E, L):
            q.X.copy_(x)
        graph.replay()
        step(E)
        torch.cuda.synchronize()
        for k, v in L.grads().items():
            assert torch.equal(v, E.grads()[k]), k
