"""The operators as a model uses them: a residual block around a relational layer, its training step with clipped gradients, captured and
replayed calls, other streams.  Numbers against the same chain in 64 bits (the layer by the CPU oracle), to the tolerance of the layers' own
tests."""
import math

import numpy as np
import pytest

from oracle import layers as O
from paper_2412_04747_amd import synth
from parity import check, TOL_F32

pytestmark = pytest.mark.gpu


def test_residual_block_training_step():
    """x -> x + rgat(norm(x)) -> + ffn(norm(.)) -> norm, its gradients, and their clipping."""
    import torch
    from paper_2412_04747_amd import autograd as A
    N, R, E, d, f = 700, 5, 6000, 64, 150
    rng, src, dst, rel, _ = synth.tiny(401, N=N, R=R, E=E)
    dst[:500] = 11
    p = synth.rgat_params(rng, N, R, d, d)
    print(f"block case N={N} R={R} E={E} d={d} f={f}", flush=True)
    g = A.Graph(N, R, src, dst, rel)
    torch.manual_seed(3)
    conv, ffn = A.RgatConv(R, d), A.GatedFfn(d, f)
    norms = [A.ResidualNorm(d) for _ in range(3)]
    for n in norms:
        torch.nn.init.normal_(n.weight, 1.0, 0.2)
    X = torch.tensor(p["X"], dtype=torch.float32, device="cuda", requires_grad=True)
    dOut = torch.tensor(p["dOut"], dtype=torch.float32, device="cuda")
    params = [q for m in (conv, ffn, *norms) for q in m.parameters()]
    y, s = norms[1](conv(g, norms[0](X)), X)
    out, s = norms[2](ffn(y), s)
    out.backward(dOut)
    grads = [q.grad.clone() for q in params]
    norm = A.clip_grad_norm_(params, 0.7)
    torch.cuda.synchronize()

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, W, ws, wt):
            ctx.save_for_backward(x, W, ws, wt)
            return torch.from_numpy(O.rgat_fwd(N, src, dst, rel, *(t.detach().numpy() for t in (x, W, ws, wt))))

        @staticmethod
        def backward(ctx, dy):
            b = O.rgat_bwd(N, src, dst, rel, *(t.detach().numpy() for t in ctx.saved_tensors), np.ascontiguousarray(dy.numpy()))
            return tuple(torch.from_numpy(b[k]) for k in ("dX", "dW", "dw_s", "dw_t"))

    q = [t.detach().cpu().double().requires_grad_() for t in (X, *params)]
    x, W, ws, wt, Wg, Wu, Wd, w0, w1, w2 = q
    nrm = lambda t, w: t / torch.sqrt((t * t).mean(1, keepdim=True) + 1e-6) * w
    s1 = Layer.apply(nrm(x, w0), W, ws, wt) + x
    y1 = nrm(s1, w1)
    a = y1 @ Wg
    want = nrm((a * torch.sigmoid(a) * (y1 @ Wu)) @ Wd + s1, w2)
    want.backward(dOut.cpu().double())
    check(out, want.detach().numpy(), TOL_F32, "out")
    check(X.grad, x.grad.numpy(), TOL_F32, "dX")
    for i, (got, t) in enumerate(zip(grads, q[1:])):
        check(got, t.grad.numpy(), TOL_F32, f"parameter {i}")
    total = math.sqrt(sum(float((t.grad ** 2).sum()) for t in q[1:]))
    assert abs(float(norm) - total) <= TOL_F32 * total and total > 0.7
    for got, t in zip(params, q[1:]):
        check(got.grad, (t.grad * (0.7 / (total + 1e-6))).numpy(), TOL_F32, "clipped")
    g.close()


def test_bf16_rows_between_layers():
    """An fp32 stream, bf16 rows into the block and gradients back: shapes, types, and each operator against its fp32 self on the same
    (rounded) values, one rounding to bf16 per stored value and two inside the block (2-norms: 2^-8 each is generous)."""
    import torch
    from paper_2412_04747_amd import autograd as A
    torch.manual_seed(5)
    N, d, f = 333, 128, 200
    stream = torch.randn(N, d, device="cuda", requires_grad=True)
    a = torch.randn(N, d, device="cuda").bfloat16().requires_grad_()
    norm, ffn = A.ResidualNorm(d, out_dtype=torch.bfloat16), A.GatedFfn(d, f, dtype=torch.bfloat16)
    y, s = norm(a, stream)
    assert y.dtype == torch.bfloat16 and s.dtype == torch.float32
    h = ffn(y)
    out, s2 = A.ResidualNorm(d, out_dtype=torch.float32)(h, s)
    dOut = torch.randn(N, d, device="cuda")
    (out * dOut).sum().backward()
    assert a.grad.dtype == torch.bfloat16 and stream.grad.dtype == torch.float32 and all(q.grad.dtype == torch.bfloat16 for q in ffn.parameters())
    assert (a.grad.float() - stream.grad).abs().max() <= 2.0 ** -8 * stream.grad.abs().max()          # the same numbers in two types
    W = [q.detach().float().requires_grad_() for q in ffn.parameters()]
    yf = y.detach().float().requires_grad_()
    hf = A.gated_ffn(yf, *W)
    assert torch.linalg.norm(h.float() - hf) <= 3 * 2.0 ** -8 * torch.linalg.norm(hf)
    dh = torch.randn(N, d, device="cuda").bfloat16()
    got = torch.autograd.grad(ffn(y.detach().requires_grad_()), list(ffn.parameters()), dh)
    want = torch.autograd.grad(hf, W, dh.float())
    for x, w in zip(got, want):
        assert torch.linalg.norm(x.float() - w) <= 3 * 2.0 ** -8 * torch.linalg.norm(w)


def test_shapes_strides_and_partial_gradients():
    import torch
    from paper_2412_04747_amd import autograd as A
    torch.manual_seed(6)
    d, f = 32, 50
    base = torch.randn(6, 7, d, device="cuda")
    w = torch.rand(d, device="cuda") + 0.5
    Wg, Wu, Wd = torch.randn(d, f, device="cuda"), torch.randn(d, f, device="cuda"), torch.randn(f, d, device="cuda")
    views = {"leading dimensions": base, "transposed": base.transpose(0, 1), "every second": base[::2], "one row": base[0, 0],
             "an offset of an element": torch.randn(5 * d + 1, device="cuda")[1:].view(5, d), "no rows": base[:0]}
    for name, v in views.items():
        flat = v.reshape(-1, d).contiguous().clone()
        assert torch.equal(A.residual_norm(v, w), A.residual_norm(flat, w).view(v.shape)), name
        assert torch.equal(A.gated_ffn(v, Wg, Wu, Wd), A.gated_ffn(flat, Wg, Wu, Wd).view(v.shape)), name
        o, s = A.residual_norm(v, w, v)
        assert torch.equal(s, v + v) and o.shape == v.shape, name
        # gradients arrive with the strides of an expanded tensor too
        x = v.detach().clone().requires_grad_()
        A.gated_ffn(x, Wg, Wu, Wd).sum().backward()
        y = flat.clone().requires_grad_()
        A.gated_ffn(y, Wg, Wu, Wd).backward(torch.ones_like(y))
        assert torch.equal(x.grad, y.grad.view(v.shape)), name
    # weights given as transposed views
    assert torch.equal(A.gated_ffn(base, Wg.t().contiguous().t(), Wu, Wd), A.gated_ffn(base, Wg, Wu, Wd))
    # what needs no gradient gets none, and the others are the same
    x, r, ww = (t.clone().requires_grad_() for t in (base, base + 1, w))
    o, s = A.residual_norm(x, ww, r)
    c = torch.randn_like(o)
    full = torch.autograd.grad((o * c).sum() + s.sum(), (x, r, ww))
    assert torch.equal(full[0], full[1])
    for i in range(3):
        t = [v.detach().requires_grad_(k == i) for k, v in enumerate((x, r, ww))]
        o, s = A.residual_norm(t[0], t[2], t[1])
        assert torch.equal(torch.autograd.grad((o * c).sum() + s.sum(), t[i])[0], full[i]), i
    o, s = A.residual_norm(x, ww, r)                     # only the sum is used
    gx, gr = torch.autograd.grad(s, (x, r), c)
    assert torch.equal(gx, c) and torch.equal(gr, c)
    o, s = A.residual_norm(x, ww, r)                     # only the norm is used
    gx, = torch.autograd.grad(o, x, c)
    assert torch.isfinite(gx).all()
    X, *W = (t.clone().requires_grad_() for t in (base, Wg, Wu, Wd))
    full = torch.autograd.grad(A.gated_ffn(X, *W), (X, *W), c)
    for i in range(4):
        t = [v.detach().requires_grad_(k == i) for k, v in enumerate((X, *W))]
        assert torch.equal(torch.autograd.grad(A.gated_ffn(*t), t[i], c)[0], full[i]), i


def test_refusals_of_the_front_end():
    import torch
    from paper_2412_04747_amd import autograd as A
    x, w = torch.randn(4, 64, device="cuda"), torch.ones(64, device="cuda")
    Wg, Wd = torch.randn(64, 20, device="cuda"), torch.randn(20, 64, device="cuda")
    for bad, kind in [(lambda: A.residual_norm(x.cpu(), w), TypeError), (lambda: A.residual_norm(x.half(), w), TypeError),
                      (lambda: A.residual_norm(x, w.bfloat16()), TypeError), (lambda: A.residual_norm(x, w[:32]), ValueError),
                      (lambda: A.residual_norm(x, w, x[:2]), ValueError), (lambda: A.gated_ffn(x, Wg, Wg, Wg), ValueError),
                      (lambda: A.gated_ffn(x.bfloat16(), Wg, Wg, Wd), TypeError), (lambda: A.gated_ffn(x, Wg, Wg, Wd, act="tanh"), ValueError),
                      (lambda: A.gated_ffn(x[:, :48], Wg[:48], Wg[:48], Wd[:, :48]), RuntimeError)]:
        with pytest.raises(kind):
            bad()
    q = torch.nn.Parameter(torch.ones(3, device="cuda"))
    q.grad = torch.ones(3, device="cuda")
    p = torch.nn.Parameter(torch.ones(3, device="cuda"))
    p.grad = torch.sparse_coo_tensor([[0]], [1.0], (3,), device="cuda")
    with pytest.raises(TypeError):
        A.clip_grad_norm_([q, p], 1.0)
    with pytest.raises(RuntimeError):                    # the same gradient twice
        A.clip_grad_norm_([q, q], 1.0)
    q.grad[1] = float("nan")
    with pytest.raises(RuntimeError):
        A.clip_grad_norm_([q], 1.0, error_if_nonfinite=True)
    assert float(q.grad[0]) == 1.0                       # nothing was scaled
    assert float(A.clip_grad_norm_([], 1.0)) == 0.0


def test_clip_takes_gradients_of_any_strides():
    import torch
    from paper_2412_04747_amd import autograd as A
    torch.manual_seed(8)
    shapes = [(30, 40), (7,), (3, 4, 5), ()]
    params = [torch.nn.Parameter(torch.zeros(s, device="cuda")) for s in shapes]
    grads = [torch.randn(40, 30, device="cuda").t(), torch.randn(21, device="cuda")[::3], torch.randn(5, 3, 4, device="cuda").permute(1, 2, 0),
             torch.randn((), device="cuda")]
    for p, g in zip(params, grads):
        p.grad = g
    want = [g.clone().double() for g in grads]
    total = math.sqrt(sum(float((g ** 2).sum()) for g in want))
    norm = A.clip_grad_norm_(iter(params + [torch.nn.Parameter(torch.zeros(2, device="cuda"))]), 1.25)
    assert abs(float(norm) - total) <= 1e-6 * total
    for p, g in zip(params, want):
        assert (p.grad.double() - g * (1.25 / (total + 1e-6))).abs().max() <= 2.0 ** -22 * g.abs().max()
    single = torch.nn.Parameter(torch.zeros(5, device="cuda"))
    single.grad = torch.full((5,), 3.0, device="cuda")
    assert abs(float(A.clip_grad_norm_(single, 1e9)) - 3.0 * math.sqrt(5.0)) < 1e-5 and (single.grad == 3.0).all()


def test_captured_and_replayed_on_another_stream():
    """A block's calls recorded into a graph and replayed over changing inputs, with eager calls of the same kind between, and a second graph
    with buffers of its own: every replay gives the eager bits."""
    import torch
    from paper_2412_04747_amd.harness import FfnLayer, GradClip, NormLayer
    rows, d, f = 300, 64, 100

    def make(seed):
        torch.manual_seed(seed)
        n, m = NormLayer(rows, d), FfnLayer(rows, d, f)
        n.x, n.residual, n.weight = torch.randn(rows, d, device="cuda"), torch.randn(rows, d, device="cuda"), torch.rand(d, device="cuda")
        m.X, m.Wg, m.Wu, m.Wd = n.out, *(torch.randn(s, device="cuda") * 0.1 for s in ((d, f), (d, f), (f, d)))
        m.dOut = n.dSum = torch.randn(rows, d, device="cuda")
        n.dOut = m.dX
        clip = GradClip([m.dWg, m.dWu, m.dWd, n.dWeight])

        def step():
            n.fwd(); m.fwd(); m.bwd(); n.bwd()
            clip.clip([m.dWg, m.dWu, m.dWd, n.dWeight], 0.5)
        return n, m, clip, step

    def results(n, m, clip):
        return [t.clone() for t in (n.sum, n.out, m.out, m.dX, m.dWg, m.dWu, m.dWd, n.dResidual, n.dWeight, clip.norm)]

    eager = make(1)
    inputs = [torch.randn(rows, d, device="cuda") for _ in range(3)]
    want = []
    for x in inputs:
        eager[0].x.copy_(x)
        eager[3]()
        want.append(results(*eager[:3]))
    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        n, m, clip, step = make(1)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
        graphs.append((graph, n, m, clip))
    for turn in range(2):
        for i, x in enumerate(inputs):
            for graph, n, m, clip in graphs:
                n.x.copy_(x)
                graph.replay()
            eager[3]()
            torch.cuda.synchronize()
            for _, n, m, clip in graphs:
                for a, b in zip(results(n, m, clip), want[i]):
                    assert torch.equal(a, b)


def test_autograd_on_another_stream():
    import torch
    from paper_2412_04747_amd import autograd as A
    torch.manual_seed(9)
    norm, ffn = A.ResidualNorm(64), A.GatedFfn(64, 100)
    x = torch.randn(500, 64, device="cuda")

    def grads():
        for q in (*norm.parameters(), *ffn.parameters()):
            q.grad = None
        y, s = norm(x, x)
        (ffn(y) + s).square().sum().backward()
        A.clip_grad_norm_([*norm.parameters(), *ffn.parameters()], 1.0)
        return [q.grad.clone() for q in (*norm.parameters(), *ffn.parameters())]

    want = grads()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = grads()
    side.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
