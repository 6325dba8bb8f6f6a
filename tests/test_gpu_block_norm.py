"""The junction of a block's output with the residual stream against its definition in 64 bits.

Tolerances, per element, in units U = 2^-24.  A mean over a row is a sum of at most 16 terms of a lane, six steps of the lanes' tree and eight wavefronts,
and a multiplication: 32 units of the terms' magnitudes.  Of n = a q1 w1, q1 takes half of that and two for the root: with three products 22.  The sum
s' = scale s + gate n adds three roundings: 25 units of |s'| := |scale s| + |gate n|, which may be A times the row's own 2-norm where the two cancel.  Then q2 is
off by 25 A + 18 units, out by 25 + 25 A + 18 + 3 <= 71 A units of q2 w2 |s'|.
Backward, the sums of the terms' magnitudes are taken: mean(g s') 25 + 34 + 1, its product with s' q2^2 by 60 + 25 + 2 (25 A + 18) + 4 <= 175 A; dT, with q2 once
more, 220 A; mean(h a) 220 A + 36, with a q1^2 and q1 three times 20 more: 330 A.  A sum over rows has the terms' 220 A + 25, and one rounding per row that a group
of lanes walks, per step of the trees and per share: 100 more.  Stored values are off by half a step of their type besides."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 1e-6
U = 2.0 ** -24
FWD, BWD, SUMS = 71, 330, 345


def _t(name):
    import torch
    return torch.bfloat16 if name == "bf16" else torch.float32


def _half(name):
    return 2.0 ** -8 if name == "bf16" else U


TYPES = [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "f32", "bf16"), ("bf16", "f32", "f32"), ("f32", "bf16", "bf16"),
         ("bf16", "f32", "bf16"), ("bf16", "bf16", "f32"), ("f32", "bf16", "f32")]
# rows, width, types, order, padding
CASES = [(1, 1, 1, "sorted", 0), (1, 64, 1, "sorted", 0), (3, 2, 2, "mixed", 0), (17, 3, 4, "sorted", 2), (5, 31, 1, "sorted", 0), (33, 32, 3, "mixed", 5),
         (1000, 64, 4, "sorted", 0), (999, 64, 4, "mixed", 60), (129, 100, 2, "sorted", 0), (64, 128, 29, "mixed", 0), (700, 128, 29, "sorted", 9), (41, 255, 1, "sorted", 0),
         (30, 349, 7, "mixed", 3), (300, 349, 7, "sorted", 20), (77, 512, 1, "sorted", 0), (9, 1000, 4, "mixed", 1), (6, 1021, 1, "sorted", 0), (40, 1020, 3, "mixed", 4),
         (12, 2036, 2, "mixed", 1), (5, 2052, 1, "sorted", 0), (3, 4099, 1, "sorted", 0), (4, 8192, 1, "sorted", 0), (2, 8191, 1, "sorted", 0), (20011, 64, 5, "sorted", 100),
         (9001, 1, 300, "mixed", 50), (6007, 16, 9, "mixed", 0),
         # several turns of every workgroup: short vectors, rows of whole workgroups
         (9000, 349, 7, "mixed", 40), (1200, 2052, 1, "sorted", 0), (1100, 1030, 3, "mixed", 17), (700, 4099, 1, "sorted", 0), (30000, 30, 3, "sorted", 11), (30000, 3, 2, "mixed", 7)]


def inputs(rows, width, types, order, pad, a, total, out, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    n = lambda *shape, scale=1.0: torch.randn(*shape, generator=g) * scale
    d = dict(a=n(rows, width) * torch.exp(0.5 * n(rows, 1)), s=n(rows, width, scale=2.0), dy=n(rows, width, scale=0.1), ds=n(rows, width, scale=0.1))
    if rows > 3:
        d["a"][1] = 0                                    # as a layer gives for a node without edges
    kind = (torch.rand(rows, generator=g) ** 1.5 * types).long().clamp(max=types - 1)
    kind = kind.sort()[0] if order == "sorted" else kind
    if pad:
        kind[rows - pad:] = torch.tensor([-1, types, 2 ** 31 - 1])[torch.arange(pad) % 3]
        for v in d.values():
            v[rows - pad:] = float("nan")
    d = {k: v.to(_t({"a": a, "s": total, "ds": total, "dy": out}[k])) for k, v in d.items()}
    d.update(kind=kind, there=(kind >= 0) & (kind < types), w_after=1.0 + n(width, scale=0.2), w_before=1.0 + n(width, scale=0.2), gate=0.5 + n(types, width, scale=0.2),
             scale=0.9 + n(types, scale=0.1))
    return d


def layer(d, types, a, total, out, without=(), held=False, flags=0, with_types=None):
    from paper_2412_04747_amd.harness import BlockNormLayer
    rows, width = d["a"].shape
    L = BlockNormLayer(rows, width, a, total, out, types, EPS, held=held, flags=flags)
    c = lambda k: None if k in without else d[k].cuda()
    L.a, L.s, L.dOut, L.dSum = c("a"), c("s"), c("dy"), c("ds")
    L.w_after, L.w_before, L.gate, L.scale = c("w_after"), c("w_before"), c("gate"), c("scale")
    if types > 1 or with_types:
        L.types = d["kind"].int().cuda()
    if L.w_before is None:
        L.dOut = None
    return L


def definition(d, types, without=(), held=None):
    """Results in 64 bits, and what their units apply to."""
    f = lambda t: t.double().numpy()
    there = d["there"].numpy()
    k = np.where(there, d["kind"].numpy(), 0)
    a, s, dy, ds = (np.where(there[:, None], f(held[q] if held and q in held else d[q]), 0.0) for q in ("a", "s", "dy", "ds"))
    if "dy" in without or "w_before" in without:
        dy = np.zeros_like(dy)
    if "ds" in without:
        ds = np.zeros_like(ds)
    width = a.shape[1]
    w1, w2 = f(d["w_after"]), f(d["w_before"])
    gate = f(d["gate"]) if "gate" not in without else np.ones((types, width))
    scale = f(d["scale"]) if "scale" not in without else np.ones(types)
    g, sc = gate[k], scale[k][:, None]
    if "w_after" in without:
        q1, w1 = np.ones((len(a), 1)), np.ones(width)
    else:
        q1 = 1.0 / np.sqrt((a * a).mean(1, keepdims=True) + EPS)
    n = a * q1 * w1
    t = sc * s + g * n
    ta = np.abs(sc * s) + np.abs(g * n)
    q2 = 1.0 / np.sqrt((t * t).mean(1, keepdims=True) + EPS)
    A = np.maximum(1.0, np.linalg.norm(ta, axis=1, keepdims=True) / np.maximum(np.linalg.norm(t, axis=1, keepdims=True), 1e-30))
    r, m = {}, {}
    r["sum"], m["sum"] = t, 25 * ta
    r["out"], m["out"] = t * q2 * w2, FWD * A * q2 * np.abs(w2) * ta
    gy = dy * w2
    dT = ds + q2 * (gy - t * q2 ** 2 * (gy * t).mean(1, keepdims=True))
    dTa = np.abs(ds) + q2 * (np.abs(gy) + ta * q2 ** 2 * (np.abs(gy) * ta).mean(1, keepdims=True))
    h, ha = g * dT * w1, np.abs(g * w1) * dTa
    if "w_after" in without:
        r["dA"], m["dA"] = h, BWD * A * ha
    else:
        r["dA"] = q1 * (h - a * q1 ** 2 * (h * a).mean(1, keepdims=True))
        m["dA"] = BWD * A * q1 * (ha + np.abs(a) * q1 ** 2 * (ha * np.abs(a)).mean(1, keepdims=True))
    r["dS"], m["dS"] = sc * dT, BWD * A * np.abs(sc) * dTa
    one = (k[None, :] == np.arange(types)[:, None]) & there[None, :]
    by = lambda v: one.astype(float) @ v
    G, Ga = by(dT * a * q1), by(A * dTa * np.abs(a) * q1)
    r["dGate"], m["dGate"] = w1 * G, SUMS * np.abs(w1) * Ga
    r["dWAfter"], m["dWAfter"] = (gate * G).sum(0), SUMS * (np.abs(gate) * Ga).sum(0)
    r["dScale"], m["dScale"] = by((dT * s).sum(1)), SUMS * by((A * dTa * np.abs(s)).sum(1))
    r["dWBefore"], m["dWBefore"] = (dy * t * q2).sum(0), SUMS * (A * np.abs(dy) * ta * q2).sum(0)
    for name in ("sum", "out", "dA", "dS"):
        r[name] = np.where(there[:, None], r[name], 0.0)
    return r, m


def within(L, d, r, m, names, types=None):
    import torch
    torch.cuda.synchronize()
    half = {"sum": L.sum, "out": L.out, "dA": L.dA, "dS": L.dS}
    for name in names:
        got = getattr(L, name).detach().cpu().double().numpy()
        h = 2.0 ** -8 if name in half and half[name].dtype == torch.bfloat16 else U
        tol = U * m[name] * 1.01 + h * np.abs(r[name]) + 2.0 ** -126
        off = np.abs(got - r[name])
        bad = ~(off <= tol)
        assert not bad.any(), f"{name}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: off {off[bad][0]:.3e}, allowed {np.broadcast_to(tol, off.shape)[bad][0]:.3e}"


ALL = ("dA", "dS", "dGate", "dWAfter", "dScale", "dWBefore")


@pytest.mark.parametrize("i,rows,width,types,order,pad", [(i, *c) for i, c in enumerate(CASES)])
def test_against_the_definition(i, rows, width, types, order, pad):
    for a, total, out in [TYPES[i % 8], TYPES[(i + 3) % 8]]:
        print(f"block_norm case rows={rows} width={width} types={types} {order} pad={pad}, {a} {total} {out}", flush=True)
        d = inputs(rows, width, types, order, pad, a, total, out, 7 * rows + width)
        L = layer(d, types, a, total, out)
        r, m = definition(d, types)
        L.fwd()
        within(L, d, r, m, ("sum", "out"))
        L.bwd()
        within(L, d, r, m, ALL)


@pytest.mark.parametrize("i,rows,width,types,order,pad", [(i, *c) for i, c in enumerate(CASES)])
def test_from_rows_in_8_bits(i, rows, width, types, order, pad):
    """The forward's codes are those of the rows themselves (zeros where a row stands for nothing); the backward is that of the values they stand for."""
    import torch
    from paper_2412_04747_amd.harness import Rows8
    a, total, out = TYPES[(i + 1) % 8]
    print(f"block_norm case in 8 bits rows={rows} width={width} types={types} {order} pad={pad}, {a} {total} {out}", flush=True)
    d = inputs(rows, width, types, order, pad, a, total, out, 3 * rows + width)
    L, whole = layer(d, types, a, total, out, held=True), layer(d, types, a, total, out)
    L.fwd()
    whole.fwd()
    assert torch.equal(L.sum, whole.sum) and torch.equal(L.out, whole.out)
    there, held = d["there"].cuda()[:, None], {}
    for name, t, got in (("a", L.a, L.held_a), ("s", L.s, L.held_s)):
        want = Rows8(rows, width)
        want.pack(torch.where(there, t, torch.zeros_like(t)))
        assert torch.equal(got.codes, want.codes) and torch.equal(got.scales, want.scales), name
        held[name] = torch.empty(rows, width, device="cuda")
        got.unpack(held[name])
        held[name] = held[name].cpu()
    r, m = definition(d, types, held=held)
    L.bwd()
    within(L, d, r, m, ALL)


@pytest.mark.parametrize("without", [("w_after",), ("gate",), ("scale",), ("w_before",), ("gate", "scale"), ("w_after", "gate"), ("w_after", "w_before"), ("ds",), ("dy",),
                                     ("w_after", "gate", "scale"), ("ds", "w_after")])
@pytest.mark.parametrize("rows,width,types", [(50, 64, 3), (33, 37, 1), (20, 1300, 2)])
def test_parts_that_are_absent(without, rows, width, types):
    print(f"block_norm case without {without} rows={rows} width={width} types={types}", flush=True)
    d = inputs(rows, width, types, "mixed", 2, "f32", "f32", "f32", 11)
    for held in (False, True):
        L = layer(d, types, "f32", "f32", "f32", without=without, held=held, with_types=True)
        kept = None
        if not {"ds", "dy"} & set(without):
            L.fwd()
        else:
            for x, to in ((L.a, L.held_a), (L.s, L.held_s)):
                if held:
                    to.pack(x)
        if held:
            import torch
            kept = {k: torch.empty(rows, width, device="cuda") for k in "as"}
            L.held_a.unpack(kept["a"])
            L.held_s.unpack(kept["s"])
            kept = {k: v.cpu() for k, v in kept.items()}
        r, m = definition(d, types, without)
        if not {"ds", "dy"} & set(without):
            within(L, d, r, m, ("sum",) if "w_before" in without else ("sum", "out"))
        r, m = definition(d, types, without, held=kept)
        L.bwd()
        names = [n for n, p in zip(ALL, ("", "", "gate", "w_after", "scale", "w_before")) if p not in without]
        within(L, d, r, m, names)


def test_one_type_given_or_not():
    """Rows of type 0 and a missing row_types are the same bits."""
    import torch
    d = inputs(300, 64, 1, "sorted", 0, "f32", "f32", "f32", 5)
    L, M = layer(d, 1, "f32", "f32", "f32"), layer(d, 1, "f32", "f32", "f32", with_types=True)
    for q in (L, M):
        q.fwd()
        q.bwd()
    for name in ("sum", "out", *ALL):
        assert torch.equal(getattr(L, name), getattr(M, name)), name


@pytest.mark.parametrize("rows,width", [(3000, 64), (40, 349), (5, 2100)])
def test_every_row_padding(rows, width):
    import torch
    from paper_2412_04747_amd import binding as B
    for flags in (0, B.RGNN_FLAG_ACCUMULATE):
        d = inputs(rows, width, 1, "sorted", 0, "f32", "f32", "f32", 6)
        d["kind"][:] = -5
        for k in ("a", "s", "dy", "ds"):
            d[k][:] = float("nan")
        L = layer(d, 1, "f32", "f32", "f32", with_types=True, flags=flags)
        results = [getattr(L, n) for n in ALL]
        for t in (L.sum, L.out, *results):
            t.fill_(2.0)
        L.fwd()
        L.bwd()
        assert not L.sum.any() and not L.out.any()
        for t in results:
            assert (t == (2.0 if flags else 0.0)).all()


@pytest.mark.parametrize("rows,width,types", [(500, 64, 3), (2, 64, 2), (41, 349, 1), (7, 2000, 2)])
def test_accumulate(rows, width, types):
    """Gradients are added to: the difference of two calls' results is within one rounding of the sum."""
    import torch
    from paper_2412_04747_amd import binding as B
    d = inputs(rows, width, types, "mixed", 1, "f32", "f32", "f32", 12)
    L, M = layer(d, types, "f32", "f32", "f32", with_types=True), layer(d, types, "f32", "f32", "f32", flags=B.RGNN_FLAG_ACCUMULATE, with_types=True)
    L.bwd()
    before = {}
    for name in ALL:
        t = getattr(M, name)
        t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(1)))
        before[name] = t.clone()
    M.bwd()
    for name in ALL:
        want = before[name].double() + getattr(L, name).double()
        assert ((getattr(M, name).double() - want).abs() <= 2 * U * (want.abs() + getattr(L, name).double().abs())).all(), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place(dtype):
    """sum and out over s and a, dA and dS over dOut and dSum, either way round: the bits of calls with buffers of their own."""
    import torch
    from paper_2412_04747_amd import binding as B
    d = inputs(700, 96, 2, "mixed", 30, dtype, dtype, dtype, 13)
    for swap in (False, True):
        L = layer(d, 2, dtype, dtype, dtype)
        L.fwd()
        L.bwd()
        a, s, dy, ds = (t.clone() for t in (L.a, L.s, L.dOut, L.dSum))
        B.rgnn_block_norm_fwd(L.desc, L._params(), a, s, a if swap else s, s if swap else a)
        torch.cuda.synchronize()
        assert torch.equal(a if swap else s, L.sum) and torch.equal(s if swap else a, L.out)
        B.rgnn_block_norm_bwd(L.desc, L._params(), L.a, L.s, None, None, dy, ds, dy if swap else ds, ds if swap else dy, None, None)
        torch.cuda.synchronize()
        assert torch.equal(dy if swap else ds, L.dA) and torch.equal(ds if swap else dy, L.dS)


def test_wanted_results_are_the_same_without_the_others():
    import torch
    from paper_2412_04747_amd import binding as B
    d = inputs(600, 64, 3, "sorted", 0, "f32", "f32", "f32", 14)
    L = layer(d, 3, "f32", "f32", "f32")
    L.bwd()
    want = {n: getattr(L, n).clone() for n in ALL}
    fields = {"dGate": "gate", "dWAfter": "w_after", "dScale": "scale", "dWBefore": "w_before"}
    for name in ALL:
        t = getattr(L, name)
        t.fill_(7.0)
        grads = B.block_norm_grads(**{fields[name]: t}) if name in fields else None
        B.rgnn_block_norm_bwd(L.desc, L._params(), L.a, L.s, None, None, L.dOut, L.dSum, t if name == "dA" else None, t if name == "dS" else None, grads,
                              L.ws if grads else None)
        torch.cuda.synchronize()
        assert torch.equal(t, want[name]), name


@pytest.mark.parametrize("rows,width,types,order", [(30000, 64, 4, "mixed"), (30000, 64, 4, "sorted"), (5000, 349, 5, "mixed")])
def test_repeated_calls_give_the_same_bits(rows, width, types, order):
    import torch
    d = inputs(rows, width, types, order, 0, "f32", "f32", "f32", 15)
    L = layer(d, types, "f32", "f32", "f32")
    L.bwd()
    want = [getattr(L, n).clone() for n in ALL]
    for _ in range(5):
        L.bwd()
        torch.cuda.synchronize()
        for n, w in zip(ALL, want):
            assert torch.equal(getattr(L, n), w), n


def test_rows_past_the_range_of_squares():
    """Rows of 1e25 (their squares are infinite in fp32) and of 1e-25, in a and in s; the other rows are not touched by an infinite one."""
    import torch
    for width in (64, 2048):
        d = inputs(12, width, 1, "sorted", 0, "f32", "f32", "f32", 16)
        d["a"][2] *= 1e25
        d["a"][3] *= 1e-25
        d["s"][4] *= 1e25
        d["s"][5] *= 1e-25
        d["a"][6] *= 1e30
        d["s"][6] *= 1e30
        L = layer(d, 1, "f32", "f32", "f32")
        r, m = definition(d, 1)
        L.fwd()
        within(L, d, r, m, ("sum", "out"))
        L.bwd()
        within(L, d, r, m, ALL)
        clean = {n: getattr(L, n).clone() for n in ("sum", "out", "dA", "dS")}
        L.a[7, 3], L.s[9, 5], L.dOut[10, 1] = float("inf"), float("nan"), float("nan")
        L.fwd()
        L.bwd()
        torch.cuda.synchronize()
        keep = torch.tensor([i not in (7, 9, 10) for i in range(12)], device="cuda")
        for n, w in clean.items():
            assert torch.equal(getattr(L, n)[keep], w[keep]), n
        assert not torch.isfinite(L.out[7]).all() and torch.isnan(L.out[9]).all() and torch.isnan(L.dA[10]).all()


def test_gradient_against_differences():
    """Central differences of the definition's loss in 64 bits along random directions, h = 1e-5: h^2 of the third derivative (some 1e3 of the terms'
    magnitudes at most, as q is of order one) is below the tolerance of the gradients."""
    import torch
    d = inputs(60, 32, 3, "mixed", 4, "f32", "f32", "f32", 17)
    L = layer(d, 3, "f32", "f32", "f32")
    L.bwd()
    torch.cuda.synchronize()
    dy, ds = (np.where(d["there"].numpy()[:, None], d[k].double().numpy(), 0.0) for k in ("dy", "ds"))

    def loss(e):
        r, _ = definition(e, 3)
        return (r["out"] * dy).sum() + (r["sum"] * ds).sum()

    _, m = definition(d, 3)
    for key, name in (("a", "dA"), ("s", "dS"), ("gate", "dGate"), ("scale", "dScale"), ("w_after", "dWAfter"), ("w_before", "dWBefore")):
        g = torch.Generator().manual_seed(3)
        for _ in range(3):
            v = torch.randn(d[key].shape, generator=g, dtype=torch.float64)
            h = 1e-5
            up, down = (loss(dict(d, **{key: d[key].double() + sign * h * v})) for sign in (1, -1))
            got = float((getattr(L, name).cpu().double() * v).sum())
            mag = U * m[name] + U * np.abs(getattr(L, name).cpu().double().numpy())
            where = np.broadcast_to(d["there"].numpy()[:, None], mag.shape) if key in "as" else np.ones(mag.shape, bool)
            tol = float((mag * np.abs(v.numpy()))[where].sum()) + 1e-7 * abs(up) / 1e-5 * 1e-4
            assert abs((up - down) / (2 * h) - got) <= tol, (name, (up - down) / (2 * h), got, tol)


@pytest.mark.parametrize("rows,width,dtype", [(17200000, 128, "bf16"), (900001, 64, "f32"), (600001, 100, "f32")])
def test_many_rows(rows, width, dtype):
    """2.2e9 elements in bf16, offsets past 32 bits; and results larger than the caches: the last rows and the first, with zeros between."""
    import torch
    from paper_2412_04747_amd.harness import BlockNormLayer
    k = 400
    print(f"block_norm case rows={rows} width={width} {dtype}, large", flush=True)
    d = inputs(2 * k, width, 1, "sorted", 0, dtype, dtype, dtype, 18)
    small = layer(d, 1, dtype, dtype, dtype, held=True)
    small.fwd()
    small.bwd()
    L = BlockNormLayer(rows, width, dtype, dtype, dtype, 1, EPS, held=True)
    L.w_after, L.w_before, L.gate, L.scale = small.w_after, small.w_before, small.gate, small.scale
    for name in ("a", "s", "dOut", "dSum"):
        t = torch.zeros(rows, width, device="cuda", dtype=_t(dtype))
        t[:k], t[-k:] = getattr(small, name)[:k], getattr(small, name)[k:]
        setattr(L, name, t)
    L.fwd()
    L.bwd()
    torch.cuda.synchronize()
    for name in ("sum", "out", "dA", "dS"):
        t, w = getattr(L, name), getattr(small, name)
        assert torch.equal(t[:k], w[:k]) and torch.equal(t[-k:], w[k:]), name
        assert not t[k:-k].any(), name
    r, m = definition(d, 1, held={n: _unpacked(h) for n, h in (("a", small.held_a), ("s", small.held_s))})
    # (more rows per lane: what is added is zeros, which round nothing)
    within(L, d, r, m, ("dGate", "dWAfter", "dScale", "dWBefore"))


def _unpacked(held):
    import torch
    t = torch.empty(held.rows, held.width, device="cuda")
    held.unpack(t)
    return t.cpu()


@pytest.mark.parametrize("rows,width,types,order", [(5000, 64, 3, "mixed"), (300, 349, 7, "sorted"), (400, 2100, 1, "sorted"), (3, 64, 2, "mixed"), (4000, 1, 315, "mixed")])
def test_nothing_is_written_past_the_buffers(rows, width, types, order):
    """Workspace, gradients, results, codes and scales of exactly the sizes asked for, inside larger buffers whose other bytes stay."""
    import torch
    from paper_2412_04747_amd import binding as B
    d = inputs(rows, width, types, order, 0, "f32", "f32", "f32", 19)
    L = layer(d, types, "f32", "f32", "f32", held=True)
    n = rows * width
    sizes = dict(ws=B.rgnn_block_norm_workspace_bytes(L.desc), sum=4 * n, out=4 * n, dA=4 * n, dS=4 * n, dWAfter=4 * width, dWBefore=4 * width, dGate=4 * types * width,
                 dScale=4 * types, ac=n, asc=rows * -(-width // 32), sc=n, ssc=rows * -(-width // 32))
    bufs = {k: torch.full((v + 1024,), 0x5A, dtype=torch.uint8, device="cuda") for k, v in sizes.items()}
    at = {k: b.data_ptr() for k, b in bufs.items()}
    a8, s8 = B.rows8(at["ac"], at["asc"]), B.rows8(at["sc"], at["ssc"])
    B.rgnn_block_norm_fwd(L.desc, L._params(), L.a, L.s, at["sum"], at["out"], a8, s8)
    B.rgnn_block_norm_bwd(L.desc, L._params(), None, None, a8, s8, L.dOut, L.dSum, at["dA"], at["dS"],
                          B.block_norm_grads(at["dWAfter"], at["dGate"], at["dScale"], at["dWBefore"]), at["ws"])
    torch.cuda.synchronize()
    for k, v in sizes.items():
        assert (bufs[k][v:] == 0x5A).all(), k
    L.fwd()
    L.bwd()
    torch.cuda.synchronize()
    for k in ("sum", "out", *ALL):
        assert torch.equal(bufs[k][:sizes[k]].view(torch.float32), getattr(L, k).flatten()), k


def test_no_rows():
    import torch
    from paper_2412_04747_amd import binding as B
    from paper_2412_04747_amd.harness import BlockNormLayer
    for flags in (0, B.RGNN_FLAG_ACCUMULATE):
        L = BlockNormLayer(0, 64, types=2, flags=flags)
        L.w_after, L.w_before = torch.ones(64, device="cuda"), torch.ones(64, device="cuda")
        L.gate, L.scale = torch.ones(2, 64, device="cuda"), torch.ones(2, device="cuda")
        L.types = torch.empty(0, dtype=torch.int32, device="cuda")
        grads = (L.dGate, L.dScale, L.dWAfter, L.dWBefore)
        for t in grads:
            t.fill_(3.0)
        L.fwd()
        L.bwd()
        torch.cuda.synchronize()
        for t in grads:
            assert (t == (3.0 if flags else 0.0)).all()


def test_captured_and_replayed_on_another_stream():
    """Two captured pairs with buffers of their own, eager calls between the replays: every replay gives the eager bits."""
    import torch
    args = (500, 64, 3, "mixed", 20, "f32", "f32", "f32")
    eager = layer(inputs(*args, 20), 3, "f32", "f32", "f32", held=True)
    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        L = layer(inputs(*args, 20), 3, "f32", "f32", "f32", held=True)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            L.fwd()
            L.bwd()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            L.fwd()
            L.bwd()
        graphs.append((graph, L))
    for turn in range(4):
        x = inputs(*args, 30 + turn)
        for _, L in [(None, eager), *graphs]:
            L.a.copy_(x["a"])
            L.types.copy_(x["kind"])
        for graph, _ in graphs:
            graph.replay()
        eager.fwd()
        eager.bwd()
        torch.cuda.synchronize()
        for _, L in graphs:
            for n in ("sum", "out", *ALL):
                assert torch.equal(getattr(L, n), getattr(eager, n)), n


# types whose places take most of a compute unit's LDS: one and several workgroups, vectors of four and of eight, rows of odd widths, types without a row
MANY_TYPES = [(700, 512, 8, "mixed", 20), (4000, 512, 8, "sorted", 30), (300, 1000, 5, "mixed", 3), (90, 1021, 7, "sorted", 2), (600, 1024, 8, "mixed", 11), (2500, 1024, 8, "sorted", 40),
              (5, 1024, 8, "mixed", 1), (9000, 128, 32, "mixed", 50), (20000, 128, 30, "sorted", 100), (60, 277, 32, "mixed", 4), (1, 600, 8, "sorted", 0)]


@pytest.mark.parametrize("dtypes", [("f32", "f32", "f32"), ("bf16", "bf16", "bf16"), ("f32", "bf16", "bf16")])
@pytest.mark.parametrize("rows,width,types,order,pad", MANY_TYPES)
def test_many_types_of_wide_rows(rows, width, types, order, pad, dtypes):
    """Forward and backward, from the rows themselves and from 8 bits, and the same bits when the backward is called again."""
    import torch
    print(f"block_norm case rows={rows} width={width} types={types} {order} pad={pad}, {dtypes}", flush=True)
    d = inputs(rows, width, types, order, pad, *dtypes, 5 * rows + width)
    held = layer(d, types, *dtypes, held=True)
    for L in (layer(d, types, *dtypes), held):
        r, m = definition(d, types)
        L.fwd()
        within(L, d, r, m, ("sum", "out"))
        if L is held:
            r, m = definition(d, types, held={"a": _unpacked(L.held_a), "s": _unpacked(L.held_s)})
        L.bwd()
        within(L, d, r, m, ALL)
        want = [getattr(L, n).clone() for n in ALL]
        L.bwd()
        torch.cuda.synchronize()
        for n, w in zip(ALL, want):
            assert torch.equal(getattr(L, n), w), n


@pytest.mark.parametrize("rows,width,dtypes,types", [(1000000, 64, ("f32", "f32", "bf16"), 4), (700001, 100, ("bf16", "bf16", "f32"), 3), (600000, 349, ("bf16", "bf16", "bf16"), 2)])
def test_results_past_the_caches(rows, width, dtypes, types):
    """Results larger than the caches with mixed types of tensors, several types of rows and padding, from the rows themselves: the bits of the first and last
    rows by themselves, zeros for the rows of zeros between them and for the padding."""
    import torch
    k = 400
    print(f"block_norm case rows={rows} width={width} types={types} {dtypes}, past the caches", flush=True)
    d = inputs(2 * k, width, types, "sorted", 30, *dtypes, 23)
    small = layer(d, types, *dtypes)
    small.fwd()
    small.bwd()
    from paper_2412_04747_amd.harness import BlockNormLayer
    L = BlockNormLayer(rows, width, *dtypes, types, EPS)
    L.w_after, L.w_before, L.gate, L.scale = small.w_after, small.w_before, small.gate, small.scale
    for name in ("a", "s", "dOut", "dSum", "types"):
        part = getattr(small, name)
        t = torch.zeros(rows, *part.shape[1:], device="cuda", dtype=part.dtype)
        t[:k], t[-k:] = part[:k], part[k:]
        if name == "types":
            t[k:-k] = part[k]                            # (in order, as the rows around are)
        setattr(L, name, t)
    for name in ("sum", "out", "dA", "dS"):
        getattr(L, name).fill_(3.0)
    L.fwd()
    L.bwd()
    torch.cuda.synchronize()
    for name in ("sum", "out", "dA", "dS"):
        t, w = getattr(L, name), getattr(small, name)
        assert torch.equal(t[:k], w[:k]) and torch.equal(t[-k:], w[k:]), name
        assert not t[k:-k].any() and not t[-30:].any(), name
    r, m = definition(d, types)
    # (more rows per lane: what is added is zeros, which round nothing)
    within(L, d, r, m, ("dGate", "dWAfter", "dScale", "dWBefore"))


def test_offsets_past_32_bits_from_the_rows_themselves():
    """2.2e9 elements in bf16, not held: the last rows and the first, with zeros between."""
    import torch
    from paper_2412_04747_amd.harness import BlockNormLayer
    rows, width, k, dtypes = 17200000, 128, 400, ("bf16", "bf16", "bf16")
    print(f"block_norm case rows={rows} width={width} bf16, large, not held", flush=True)
    d = inputs(2 * k, width, 1, "sorted", 0, *dtypes, 24)
    small = layer(d, 1, *dtypes)
    small.bwd()
    L = BlockNormLayer(rows, width, *dtypes, 1, EPS)
    L.w_after, L.w_before, L.gate, L.scale = small.w_after, small.w_before, small.gate, small.scale
    for name in ("a", "s", "dOut", "dSum"):
        t = torch.zeros(rows, width, device="cuda", dtype=torch.bfloat16)
        t[:k], t[-k:] = getattr(small, name)[:k], getattr(small, name)[k:]
        setattr(L, name, t)
    L.bwd()
    torch.cuda.synchronize()
    for name in ("dA", "dS"):
        t, w = getattr(L, name), getattr(small, name)
        assert torch.equal(t[:k], w[:k]) and torch.equal(t[-k:], w[k:]), name
        assert not t[k:-k].any(), name
    r, m = definition(d, 1)
    within(L, d, r, m, ("dGate", "dWAfter", "dScale", "dWBefore"))
