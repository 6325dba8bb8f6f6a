"""Feed-forward block in bf16: results are those of the definition in 64 bits rounded once, whatever the number of rows.

A result may be off by half a unit in the last place of bf16, of the binade that its value lies in, and by what the kernel's own arithmetic leaves: the
bound of `test_gpu_ffn` with act(g) u and the gradients of g and u held to 16 bits (two planes of 8, rounded to nearest: 2^-16 relative).  Of that the
smaller of two: every rounding at its worst, or eight times what as many independent ones add up to."""
import numpy as np
import pytest

from test_gpu_ffn import U, Val, _inputs, _layer, add, mm, times

pytestmark = pytest.mark.gpu
HELD = 2.0 ** -16


def unrounded(p, act):
    X, Wg, Wu, Wd, dY = (Val(p[k].double().numpy()) for k in ("X", "Wg", "Wu", "Wd", "dOut"))
    rows, d, f = X.v.shape[0], X.v.shape[1], Wg.v.shape[1]
    kd, kf, kn = d // 16 + 4, 2 * (2 * ((f + 31) // 32)) + 4, 2 * 2 * ((rows + 31) // 32) + 4        # (two instructions where an operand has two planes)
    g, u, dh = mm(X, Wg, kd), mm(X, Wu, kd), mm(dY, Wd.T, kd)
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-g.v))
        n = (8 + np.abs(g.v)) * U              # (the exponent, g times a rounded constant, is off by half a unit of |g| twice)
        a = Val(g.v * s, 1.1 * g.e + n * np.abs(g.v * s), 1.1 * g.r + n * np.abs(g.v * s))
        slope = Val(s * (1 + g.v * (1 - s)), 0.5 * g.e + n * (1 + np.abs(g.v)), 0.5 * g.r + n * (1 + np.abs(g.v)))
    else:
        a, slope = Val(np.maximum(g.v, 0.0), g.e, g.r), Val((g.v > 0).astype(np.float64))
    h, du, dg = times(a, u).half(HELD), times(dh, a).half(HELD), times(times(dh, u), slope).half(HELD)
    return {"out": mm(h, Wd, kf), "dX": add(mm(dg, Wg.T, kf), mm(du, Wu.T, kf)), "dWg": mm(X.T, dg, kn), "dWu": mm(X.T, du, kn), "dWd": mm(h.T, dY, kn)}


def half_unit(v):
    """Half a unit in the last place of bf16 (8 significant bits) at v."""
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - 8)


# one row, few rows, and rows for which the weights are laid out, with chunks divided among four, two and one group of wavefronts
SIZES = [(1, 128, 512), (37, 64, 256), (900, 128, 341), (3001, 64, 256), (9001, 64, 130), (3001, 128, 341), (20003, 64, 200), (20003, 128, 256), (40001, 32, 200)]


@pytest.mark.parametrize("rows,width,hidden", SIZES)
@pytest.mark.parametrize("act", ["silu", "relu"])
def test_one_rounding(rows, width, hidden, act):
    import torch
    print(f"ffn case rows={rows} width={width} hidden={hidden} bf16 {act}", flush=True)
    p = _inputs(rows, width, hidden, "bf16", act, rows + hidden)
    L = _layer(p, act)
    L.fwd(); L.bwd()
    torch.cuda.synchronize()
    want = unrounded(p, act)
    for k, got in (("out", L.out), *L.grads().items()):
        off, w = np.abs(got.cpu().double().numpy() - want[k].v), want[k]
        left = np.minimum(w.e, 8 * w.r)
        tol = half_unit(np.abs(w.v) + left) + left + 1e-30           # (of the next binade where the error carries the value across)
        bad = ~(off <= tol)
        assert not bad.any(), f"{k}: {bad.sum()} of {bad.size}, first at {np.argwhere(bad)[0]}: off {off[bad][0]:.3e}, allowed {tol[bad][0]:.3e}"


def test_a_row_has_the_same_output_among_few_and_many():
    """The same nodes scored alone, among a mini-batch's and among all.  What 16 bits leave, at most 2^-16 of sum |h| |Wd| on either side, moves a
    value across a border between two results as often as it is a share of the step between them; then by one step."""
    import torch
    p = _inputs(40000, 64, 256, "bf16", "silu", 5)
    X, Wg, Wu, Wd = (p[k].double() for k in ("X", "Wg", "Wu", "Wd"))
    size = ((torch.nn.functional.silu(X @ Wg) * (X @ Wu)).abs() @ Wd.abs()).numpy()
    outs = []
    for rows in (4, 300, 3000, 12000, 40000):
        print(f"ffn case rows={rows} width=64 hidden=256 bf16", flush=True)
        L = _layer({k: v[:rows] if k in ("X", "dOut") else v for k, v in p.items()}, "silu")
        L.fwd()
        outs.append(L.out.cpu().double().numpy())
    for a, b in zip(outs, outs[1:]):
        b = b[:len(a)]
        step, moved = 2 * half_unit(np.maximum(np.abs(a), np.abs(b))), 2 * HELD * size[:len(a)]
        off, often = np.abs(a - b), np.minimum(1.0, moved / step)
        assert (off <= step + moved).all(), len(a)
        assert (off > 0).sum() <= often.sum() + 4 * np.sqrt(often.sum()) + 2, len(a)
