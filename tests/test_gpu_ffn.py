"""Gated feed-forward block against its definition in 64 bits.

Tolerances.  A product of n terms in fp32 is off by at most k roundings of the sum of the terms' magnitudes, where k counts the roundings of
the running sum: one per matrix instruction, n / 16 of them (six times that for three planes), and a few in front and behind.  So the bound of a
product C = A B with errors E_A, E_B of its operands is  k 2^-24 |A||B| + E_A |B| + |A| E_B, carried through the formulas below.  silu and its
slope are right to 8 units of 2^-24 (exponential, sum, reciprocal, three products; the slope of the slope is at most 0.5, of silu 1.1).
Rounded operands (bf16) and stored results add half a step, 2^-8 of their magnitude for bf16.  Besides that bound per element, which
no error may exceed, roundings are as good as independent: the 2-norm of all errors has to be within the 2-norm of the bound with 4 sqrt(k) for k."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _inputs(rows, d, f, dtype, act, seed):
    """fp32 or bf16 tensors on the CPU.  For relu quarters of small integers: products and sums are exact, so that the sign of g,
    which decides over a gradient, does not hang on a rounding."""
    import torch
    g = torch.Generator().manual_seed(seed)
    if act == "relu":
        n = lambda scale, *s: torch.randint(-4, 5, s, generator=g).float() / 4
    else:
        n = lambda scale, *s: torch.randn(*s, generator=g) * scale
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    return {"X": n(1.0, rows, d).to(t), "Wg": n(d ** -0.5, d, f).to(t), "Wu": n(d ** -0.5, d, f).to(t), "Wd": n(f ** -0.5, f, d).to(t),
            "dOut": n(0.1, rows, d).to(t)}


def _layer(p, act, flags=0):
    from paper_2412_04747_amd.harness import FfnLayer
    import torch
    dtype = "bf16" if p["X"].dtype == torch.bfloat16 else "f32"
    L = FfnLayer(p["X"].shape[0], p["X"].shape[1], p["Wg"].shape[1], dtype, act, flags=flags)
    for k, v in p.items():
        setattr(L, k, v.cuda())
    return L


class Val:
    """A value in 64 bits, its error bound, and the same with independent roundings."""

    def __init__(self, v, e=0.0, r=0.0):
        self.v, self.e, self.r = v, np.broadcast_to(e, v.shape), np.broadcast_to(r, v.shape)

    def half(self, step):
        return Val(self.v, self.e + np.abs(self.v) * step, np.hypot(self.r, np.abs(self.v) * step))

    @property
    def T(self):
        return Val(self.v.T, self.e.T, self.r.T)


def mm(a, b, k):
    A, Bm = np.abs(a.v), np.abs(b.v)
    size = A @ Bm
    root = lambda x, y: np.sqrt((x * x) @ (y * y))        # independent errors of the operands
    return Val(a.v @ b.v, k * U * size + a.e @ Bm + A @ b.e,
               4 * np.sqrt(k) * U * root(A, Bm) + root(a.r, Bm) + root(A, b.r))


def times(a, b, k=1):
    v = a.v * b.v
    return Val(v, np.abs(a.v) * b.e + a.e * np.abs(b.v) + a.e * b.e + k * U * np.abs(v),
               np.abs(a.v) * b.r + a.r * np.abs(b.v) + k * U * np.abs(v))


def add(a, b):
    return Val(a.v + b.v, a.e + b.e + U * np.abs(a.v + b.v), np.hypot(a.r, b.r) + U * np.abs(a.v + b.v))


def expected(p, act, dtype):
    bf = dtype == "bf16"
    step = 2.0 ** -8 if bf else U
    six = 1 if bf else 6
    X, Wg, Wu, Wd, dY = (Val(p[k].double().numpy()) for k in ("X", "Wg", "Wu", "Wd", "dOut"))
    rows, d, f = X.v.shape[0], X.v.shape[1], Wg.v.shape[1]
    kd, kf, kn = six * (d // 16) + 4, six * (2 * ((f + 31) // 32)) + 4, six * 2 * ((rows + 31) // 32) + 4
    g, u, dh = mm(X, Wg, kd), mm(X, Wu, kd), mm(dY, Wd.T, kd)
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-g.v))
        a = Val(g.v * s, 1.1 * g.e + 8 * U * np.abs(g.v * s), 1.1 * g.r + 8 * U * np.abs(g.v * s))
        slope = Val(s * (1 + g.v * (1 - s)), 0.5 * g.e + 8 * U * (1 + np.abs(g.v)), 0.5 * g.r + 8 * U * (1 + np.abs(g.v)))
    else:
        a, slope = Val(np.maximum(g.v, 0.0), g.e, g.r), Val((g.v > 0).astype(np.float64))
    op = lambda t: t.half(step) if bf else t.half(2.0 ** -26)
    h, du, dg = op(times(a, u)), op(times(dh, a)), op(times(times(dh, u), slope))
    return {"out": mm(h, Wd, kf).half(step), "dX": add(mm(dg, Wg.T, kf), mm(du, Wu.T, kf)).half(step), "dWg": mm(X.T, dg, kn).half(step),
            "dWu": mm(X.T, du, kn).half(step), "dWd": mm(h.T, dY, kn).half(step)}


def _check(got, want, what):
    got = got.detach().cpu().double().numpy()
    off = np.abs(got - want.v)
    tol = want.e + 1e-30
    bad = ~(off <= tol)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: off {off[bad][0]:.3e}, allowed {tol[bad][0]:.3e}"
    n, m = np.linalg.norm(off), np.linalg.norm(want.r + 1e-30)
    print(f"  {what}: 2-norm of the errors {n:.2e}, allowed {m:.2e}, of the values {np.linalg.norm(want.v):.2e}", flush=True)
    assert n <= m, what


CASES = [(1, 32, 1), (1, 128, 512), (2, 64, 33), (3, 128, 2500), (4, 32, 97), (4, 64, 300), (5, 128, 70), (31, 64, 31), (33, 32, 32), (127, 128, 65), (129, 64, 86), (300, 128, 341), (1000, 32, 86),
         (1000, 128, 128), (513, 64, 1000), (4099, 64, 256)]


@pytest.mark.parametrize("rows,width,hidden", CASES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_against_the_definition(rows, width, hidden, dtype, act):
    import torch
    print(f"ffn case rows={rows} width={width} hidden={hidden} {dtype} {act}", flush=True)
    p = _inputs(rows, width, hidden, dtype, act, rows + width + hidden)
    L = _layer(p, act)
    L.fwd(); L.bwd()
    torch.cuda.synchronize()
    want = expected(p, act, dtype)
    _check(L.out, want["out"], "out")
    for k, v in L.grads().items():
        _check(v, want[k], k)


@pytest.mark.parametrize("rows,width,hidden,dtype", [(3001, 64, 130, "bf16"), (9001, 64, 33, "bf16"), (9001, 64, 200, "bf16"), (3001, 128, 40, "bf16"),
                                                     (5003, 64, 97, "f32"), (12001, 64, 90, "f32"), (9003, 128, 65, "f32"), (33001, 32, 97, "f32"),
                                                     (70001, 128, 40, "bf16"), (70001, 64, 96, "bf16"), (70001, 32, 200, "bf16"), (40003, 64, 70, "f32"),
                                                     (40003, 128, 33, "f32")])
def test_many_rows(rows, width, hidden, dtype):
    """Sizes at which the weights are laid out first: chunks divided among four, two and one group of wavefronts, in even and uneven numbers."""
    import torch
    print(f"ffn case rows={rows} width={width} hidden={hidden} {dtype}", flush=True)
    p = _inputs(rows, width, hidden, dtype, "silu", 3)
    L = _layer(p, "silu")
    L.fwd(); L.bwd()
    torch.cuda.synchronize()
    want = expected(p, "silu", dtype)
    _check(L.out, want["out"], "out")
    for k, v in L.grads().items():
        _check(v, want[k], k)


def test_gradient_against_differences():
    """Gradients of the kernels (fp32) against central differences of the definition in 64 bits."""
    import torch
    p = _inputs(9, 32, 45, "f32", "silu", 21)
    L = _layer(p, "silu")
    L.bwd()
    torch.cuda.synchronize()
    q = {k: v.double() for k, v in p.items()}

    def loss(q):
        g = q["X"] @ q["Wg"]
        return float(((g * torch.sigmoid(g) * (q["X"] @ q["Wu"])) @ q["Wd"] * q["dOut"]).sum())

    h = 1e-6
    for name, at in (("X", (0, 0)), ("X", (8, 31)), ("Wg", (3, 44)), ("Wg", (31, 0)), ("Wu", (5, 6)), ("Wd", (44, 31)), ("Wd", (0, 7))):
        up, dn = dict(q), dict(q)
        up[name], dn[name] = q[name].clone(), q[name].clone()
        up[name][at] += h
        dn[name][at] -= h
        # values of order 0.1, 1e-16 / h off by the differences, 1e-6 of the value by fp32
        assert abs((loss(up) - loss(dn)) / (2 * h) - float(L.grads()["d" + name][at])) < 1e-6, (name, at)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_repeatable_bounded_and_alone(dtype):
    """The same bits twice; nothing written behind the last row or the workspace; a row with NaN touches no other row."""
    import torch
    from paper_2412_04747_amd import binding as B
    for rows, width, hidden in ((45, 64, 100), (1, 128, 77), (700, 32, 250)):
        print(f"ffn case rows={rows} width={width} hidden={hidden} {dtype}", flush=True)
        p = _inputs(rows, width, hidden, dtype, "silu", 31)
        L = _layer(p, "silu")
        L.fwd(); L.bwd()
        first = [t.clone() for t in (L.out, *L.grads().values())]
        t = L.out.dtype
        big = torch.full((2, rows + 40, width), 7.0, device="cuda", dtype=t)
        f, b = B.rgnn_ffn_workspace_bytes(L.desc)
        ws = torch.full((max(f, b) + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
        L.out, L.dX, L.ws = big[0, :rows], big[1, :rows], ws
        L.fwd()
        assert (ws[f:] == 0xA5).all()
        L.bwd()
        assert (ws[max(f, b):] == 0xA5).all() and (big[:, rows:] == 7.0).all()
        for x, y in zip(first, (L.out, *L.grads().values())):
            assert torch.equal(x, y)
        if rows > 1:
            L.X[rows // 2, 3] = float("nan")
            L.X[0, 0] = float("inf")
            L.fwd(); L.bwd()
            good = [i for i in range(rows) if i not in (0, rows // 2)]
            assert torch.equal(L.out[good], first[0][good]) and torch.equal(L.dX[good], first[1][good])
            assert not L.out[rows // 2].isfinite().any() and not L.out[0].isfinite().any()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [33, 3000, 20003])
def test_accumulate_and_optional_results(rows, dtype):
    """Gradients added to what is there; a result that is not asked for leaves the others' bits."""
    import torch
    from paper_2412_04747_amd import binding as B
    print(f"ffn case rows={rows} {dtype}", flush=True)
    p = _inputs(rows, 64, 80, dtype, "silu", 41)
    L, M = _layer(p, "silu"), _layer(p, "silu", B.RGNN_FLAG_ACCUMULATE)
    L.bwd()
    for t in M.grads().values():
        t.fill_(1.0)
    M.bwd()
    step = 2.0 ** -8 if dtype == "bf16" else U
    for k, v in L.grads().items():
        # a = round(v + 1), b = round(v): half a step of either; fp32 may add in another order, one more
        v = v.double()
        assert ((M.grads()[k].double() - 1.0 - v).abs() <= 3.1 * step * (1 + v.abs())).all(), k
    want = {k: v.clone() for k, v in L.grads().items()}
    for t in L.grads().values():
        t.zero_()
    B.rgnn_ffn_bwd(L.desc, L.X, L.Wg, L.Wu, L.Wd, L.dOut, None, L.dWg, L.dWu, L.dWd, L.ws)
    assert (L.dX == 0).all() and all(torch.equal(v, want[k]) for k, v in L.grads().items() if k != "dX")
    for t in L.grads().values():
        t.zero_()
    B.rgnn_ffn_bwd(L.desc, L.X, L.Wg, L.Wu, L.Wd, L.dOut, L.dX, None, None, None, L.ws)
    assert torch.equal(L.dX, want["dX"]) and (L.dWg == 0).all() and (L.dWd == 0).all()
    B.rgnn_ffn_bwd(L.desc, L.X, L.Wg, L.Wu, L.Wd, L.dOut, None, None, None, None, L.ws)


def test_no_rows():
    from paper_2412_04747_amd import binding as B
    import torch
    from paper_2412_04747_amd.harness import FfnLayer
    N = FfnLayer(0, 64, 20)
    N.X = N.dOut = torch.empty(0, 64, device="cuda")
    N.Wg, N.Wu, N.Wd = (torch.ones(s, device="cuda") for s in ((64, 20), (64, 20), (20, 64)))
    N.dWg.fill_(2.0)
    N.fwd(); N.bwd()
    assert (N.dWg == 0).all() and (N.dWu == 0).all() and (N.dWd == 0).all()
    N.desc.flags = B.RGNN_FLAG_ACCUMULATE
    N.dWu.fill_(2.0)
    N.bwd()
    assert (N.dWu == 2).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_widest_hidden(dtype):
    """512 chunks, few rows and many."""
    import torch
    for rows in (40, 33000):
        print(f"ffn case rows={rows} width=32 hidden=16384 {dtype}", flush=True)
        p = _inputs(40, 32, 16384, dtype, "silu", 61)
        n = (rows + 39) // 40
        p["X"], p["dOut"] = p["X"].repeat(n, 1)[:rows], torch.cat([p["dOut"], torch.zeros(40 * (n - 1), 32).to(p["dOut"].dtype)])[:rows]
        L = _layer(p, "silu")
        L.fwd(); L.bwd()
        torch.cuda.synchronize()
        # rows 40 and on repeat the first forty, with a gradient of zeros
        want = expected({k: v[:40] if k in ("X", "dOut") else v for k, v in p.items()}, "silu", dtype)
        _check(L.out[:40], want["out"], "out")
        assert torch.equal(L.out, L.out[:40].repeat(n, 1)[:rows])
        for k, v in L.grads().items():
            _check(v[:40] if k == "dX" else v, want[k], k)
        assert (L.dX[40:] == 0).all()


def test_extreme_gates():
    """Gates far out: silu is 0 or the gate itself, its slope 0 or 1; no NaN from the exponential's overflow."""
    import torch
    rows, d, f = 64, 32, 32
    p = _inputs(rows, d, f, "f32", "silu", 51)
    p["Wg"] = torch.eye(d)
    p["X"] = torch.where(p["X"] > 0, 200.0, -200.0) * (1 + p["X"].abs())
    L = _layer(p, "silu")
    L.fwd(); L.bwd()
    want = expected(p, "silu", "f32")
    _check(L.out, want["out"], "out")
    for k, v in L.grads().items():
        _check(v, want[k], k)


def test_more_than_32_bits_of_elements():
    """Rows past 2^31 elements: the same as those rows alone."""
    import torch
    from paper_2412_04747_amd.harness import FfnLayer
    rows, width, hidden = (1 << 24) + 37, 128, 16
    print(f"ffn case rows={rows} width={width} hidden={hidden} bf16", flush=True)
    L = FfnLayer(rows, width, hidden, "bf16")
    L.X = torch.empty(rows, width, device="cuda", dtype=torch.bfloat16).normal_()
    L.Wg, L.Wu = (torch.randn(width, hidden, device="cuda").mul_(0.1).bfloat16() for _ in range(2))
    L.Wd = torch.randn(hidden, width, device="cuda").mul_(0.1).bfloat16()
    L.fwd()
    L.dOut = L.out
    L.bwd()
    n = 70001                                            # (as many as make the same plan)
    tail = FfnLayer(n, width, hidden, "bf16")
    tail.X, tail.Wg, tail.Wu, tail.Wd = L.X[-n:].clone(), L.Wg, L.Wu, L.Wd
    tail.fwd()
    tail.dOut = tail.out
    tail.bwd()
    assert torch.equal(L.out[-n:], tail.out) and torch.equal(L.dX[-n:], tail.dX)
