"""Feed-forward block in fp32 with many hidden values: the errors of out and dX do not grow with every matrix instruction of a row.

32 hidden values' products are summed on their own (their roundings are of their own magnitude, sqrt(chunks) below the result's) and then added:
`chunks` roundings of a sum that grows to the result's.  A rounding is off by half a unit at most, U of the value, half that in the mean square or less, and
roundings are independent: 0.5 sqrt(chunks) U of the result's 2-norm.  To that the hidden values' own errors, 28 roundings of g and u (four steps of 16
columns, six products each), 8 of the activation, and the chunks' 12: within 12 U in the mean square, wherever the hidden values' errors are independent."""
import math

import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.mark.parametrize("rows,width,hidden", [(33000, 64, 16384), (20000, 64, 8192), (9000, 128, 8192), (13000, 32, 16384)])
def test_errors_of_many_hidden_values(rows, width, hidden):
    import torch
    from paper_2412_04747_amd.harness import FfnLayer
    print(f"ffn case rows={rows} width={width} hidden={hidden} f32", flush=True)
    g = torch.Generator(device="cuda").manual_seed(3)
    n = lambda scale, *s: torch.randn(*s, generator=g, device="cuda") * scale
    L = FfnLayer(rows, width, hidden)
    L.X, L.dOut = n(1.0, rows, width), n(0.1, rows, width)
    L.Wg, L.Wu, L.Wd = n(width ** -0.5, width, hidden), n(width ** -0.5, width, hidden), n(hidden ** -0.5, hidden, width)
    L.fwd(); L.bwd()
    m = 500                                              # the last rows
    X, dY, Wg, Wu, Wd = (t.double() for t in (L.X[-m:], L.dOut[-m:], L.Wg, L.Wu, L.Wd))
    a, u, dh = X @ Wg, X @ Wu, torch.mm(dY, Wd.t().contiguous())
    s = torch.sigmoid(a)
    want = {"out": (a * s * u) @ Wd,
            "dX": torch.mm(dh * u * s * (1 + a * (1 - s)), Wg.t().contiguous()) + torch.mm(dh * a * s, Wu.t().contiguous())}
    allowed = (0.5 * math.sqrt((hidden + 31) // 32) + 12) * U
    for k, got in (("out", L.out), ("dX", L.dX)):
        off = float((got[-m:].double() - want[k]).norm() / want[k].norm())
        print(f"  {k}: {off:.2e}, allowed {allowed:.2e}", flush=True)
        assert off <= allowed, k
