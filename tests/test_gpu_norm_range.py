"""Residual norm of rows whose squares, or their sum, leave the range of fp32.  Bounds as in `test_gpu_row_norm`, relative; results below 2^-126 are
held to multiples of 2^-149, and a product of such to a few of them; bf16, with 7 bits behind the point for fp32's 23, holds multiples of 2^-126-7 = 2^-133
there, so that its rounding is off by up to 2^-134."""
import numpy as np
import pytest

from test_gpu_row_norm import U, _half, _within

pytestmark = pytest.mark.gpu
EPS = 1e-6
TINY = {"f32": 8 * 2.0 ** -149, "bf16": 2.0 ** -134 + 8 * 2.0 ** -149}


@pytest.mark.parametrize("width", [1, 3, 32, 64, 128, 349, 1000, 1024, 2052, 4099, 8192])
@pytest.mark.parametrize("x,out", [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16")])
def test_large_rows_among_others(width, x, out):
    import torch
    from paper_2412_04747_amd.harness import NormLayer
    rows = 2101 if width <= 128 else 53
    print(f"norm case rows={rows} width={width} types {x} {out}", flush=True)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}
    g = torch.Generator().manual_seed(width)
    n = lambda scale, kind: (torch.randn(rows, width, generator=g) * scale).to(t[kind])
    X = n(1.0, "f32")
    X[3::7] *= 3e17                                      # the sum leaves the range where the row is wide
    X[5::7] *= 1e25                                      # every square does
    X[6::7, width // 2] = 2e20                           # one does
    X[2] = 3.3e38 * torch.sign(X[2])                     # as large as there is
    X = X.to(t[x])
    assert X.isfinite().all()
    w, dy, ds = 1.0 + 0.2 * torch.randn(width, generator=g), n(0.1, out), None
    L = NormLayer(rows, width, x, x, out, EPS, residual=False)
    L.x, L.weight, L.dOut = X.cuda(), w.cuda(), dy.cuda()
    L.sum = L.x
    L.fwd(); L.bwd()
    torch.cuda.synchronize()
    s, w, dy = X.double().numpy(), w.double().numpy(), dy.double().numpy()
    q = 1.0 / np.sqrt((s * s).mean(1, keepdims=True) + EPS)
    want = s * q * w
    _within(L.out, want, np.abs(want) * (_half(out) + 32 * U) + TINY[out], "out")
    gy = dy * w
    along = q * q * (gy * s).mean(1, keepdims=True)
    dx = q * (gy - s * along)
    size = q * (np.abs(gy) + np.abs(s) * q * q * np.abs(gy * s).mean(1, keepdims=True))
    _within(L.dX, dx, np.abs(dx) * _half(x) + size * 48 * U + TINY[x], "dX")
    _within(L.dWeight, (dy * s * q).sum(0), np.abs(dy * s * q).sum(0) * (64 + rows / 512) * U + rows * TINY["f32"], "dWeight")


def test_residual_of_large_rows():
    """The sum is stored as it is, not scaled; the gradient that reaches it on its other way is added as it is."""
    import torch
    from paper_2412_04747_amd.harness import NormLayer
    rows, width = 40, 2052
    g = torch.Generator().manual_seed(1)
    n = lambda scale: torch.randn(rows, width, generator=g) * scale
    x, r, w, dy, ds = n(1e18), n(2e18), 1.0 + 0.2 * torch.randn(width, generator=g), n(0.1), n(1e-19)
    L = NormLayer(rows, width, eps=EPS)
    L.x, L.residual, L.weight, L.dOut, L.dSum = x.cuda(), r.cuda(), w.cuda(), dy.cuda(), ds.cuda()
    L.fwd(); L.bwd()
    assert torch.equal(L.sum.cpu(), x + r)
    s, w, dy, ds = (x + r).double().numpy(), w.double().numpy(), dy.double().numpy(), ds.double().numpy()
    q = 1.0 / np.sqrt((s * s).mean(1, keepdims=True) + EPS)
    _within(L.out, s * q * w, np.abs(s * q * w) * 33 * U, "out")
    gy = dy * w
    dx = ds + q * (gy - s * q * q * (gy * s).mean(1, keepdims=True))
    size = np.abs(ds) + q * (np.abs(gy) + np.abs(s) * q * q * np.abs(gy * s).mean(1, keepdims=True))
    _within(L.dResidual, dx, np.abs(dx) * U + size * 48 * U, "dResidual")
