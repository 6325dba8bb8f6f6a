"""Global gradient norm and clipping against their definition in 64 bits.  The norm is formed in fp64 and stored in fp32: half a step, 2^-24.  A
clipped value is the gradient times the coefficient rounded to fp32: two roundings, 2^-23, and the storage's half step for bf16."""
import math

import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


def _grads(shapes, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    return [(torch.randn(*s, generator=g) * 10.0 ** -(i % 4)).to(torch.bfloat16 if bf else torch.float32).cuda() for i, (s, bf) in enumerate(shapes)]


def _check(before, after, norm, max_norm):
    import torch
    want = math.sqrt(sum(float(g.double().pow(2).sum()) for g in before))
    assert abs(float(norm) - want) <= want * 1.01 * U
    c = min(1.0, max_norm / (want + 1e-6))
    for i, (b, a) in enumerate(zip(before, after)):
        tol = b.double().abs() * c * ((2.0 ** -8 if b.dtype == torch.bfloat16 else 0.0) + 2.1 * U) + 1e-40
        if c == 1.0:
            assert torch.equal(a, b), i
        else:
            assert ((a.double() - b.double() * c).abs() <= tol).all(), i


SETS = [[((1,), False)], [((64, 64), False)] * 3, [((0,), False), ((5, 7), True), ((1,), False), ((0, 3), True)], [((4097,), True), ((12289,), False)],
        [((3, i + 1), i % 3 == 0) for i in range(300)], [((1000003,), False), ((777, 1001), True), ((64,), False)]]


@pytest.mark.parametrize("i", range(len(SETS)))
@pytest.mark.parametrize("share", [0.0, 0.3, 3.0, math.inf])
@pytest.mark.parametrize("in_place", [True, False])
def test_against_the_definition(i, share, in_place):
    import torch
    from paper_2412_04747_amd.harness import GradClip
    print(f"clip case set {i} share {share} in_place={in_place}", flush=True)
    grads = _grads(SETS[i], i)
    before = [g.clone() for g in grads]
    norm = math.sqrt(sum(float(g.double().pow(2).sum()) for g in grads))
    L = GradClip(grads, in_place)
    L.clip(grads, share * norm if share < math.inf else share)
    torch.cuda.synchronize()
    _check(before, grads if in_place else L.clipped, L.norm, share * norm if share < math.inf else share)
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(before, grads))


def test_slices_of_any_alignment():
    """Gradients that are slices of one buffer, at every offset of elements, next to each other; what lies between them stays."""
    import torch
    from paper_2412_04747_amd.harness import GradClip
    for dtype in (torch.float32, torch.bfloat16):
        flat = torch.randn(100000, device="cuda").to(dtype)
        cuts = [0, 1, 6, 17, 4113, 8300, 8300 + 16384, 50001]
        parts = [flat[a:b] for a, b in zip(cuts[:-1], cuts[1:])]
        before, rest = [p.clone() for p in parts], flat[cuts[-1]:].clone()
        L = GradClip(parts)
        L.clip(parts, 1.5)
        _check(before, parts, L.norm, 1.5)
        assert torch.equal(rest, flat[cuts[-1]:])
        # the same elements as one tensor: the same norm up to its own rounding
        M = GradClip([torch.cat(before)])
        M.clip([torch.cat(before)], 1.5)
        assert abs(float(M.norm) - float(L.norm)) <= 2 * U * float(M.norm)


def test_extreme_values():
    import torch
    from paper_2412_04747_amd.harness import GradClip

    def clip(values, max_norm):
        g = [torch.tensor(values, device="cuda"), torch.ones(5, device="cuda")]
        L = GradClip(g)
        L.clip(g, max_norm)
        return float(L.norm), g

    n, g = clip([3e38, 1e30], 1.0)                       # the squares are in fp64
    assert abs(n - 3e38) <= 3e38 * 2 * U and abs(float(g[0][0]) - 1.0) <= 2 * 2 * U and float(g[1][0]) > 0
    n, g = clip([1e-30, 2e-30], 1.0)
    assert abs(n - math.sqrt(5.0)) < 1e-6 and (g[1] - 1 / math.sqrt(5.0)).abs().max() < 1e-6
    n, g = clip([float("inf"), 1.0], 1.0)
    assert n == math.inf and math.isnan(float(g[0][0])) and float(g[0][1]) == 0.0 and (g[1] == 0).all()
    n, g = clip([float("nan"), 1.0], 1.0)
    assert math.isnan(n) and all(t.isnan().all() for t in g)
    n, g = clip([float("inf"), 1.0], math.inf)
    assert n == math.inf and float(g[0][1]) == 1.0 and (g[1] == 1).all()
    zero = [torch.zeros(100, device="cuda")]
    L = GradClip(zero)
    L.clip(zero, 0.0)
    assert float(L.norm) == 0.0 and (zero[0] == 0).all()
    none = GradClip([])
    none.clip([], 1.0)
    assert float(none.norm) == 0.0


def test_norm_alone_and_repeatable():
    import torch
    from paper_2412_04747_amd import binding as B
    from paper_2412_04747_amd.harness import GradClip
    grads = _grads(SETS[5], 3)
    L = GradClip(grads, in_place=False)
    L.clip(grads, 0.5)
    first, norm = [t.clone() for t in L.clipped], L.norm.clone()
    L.clip(grads, 0.5)
    assert torch.equal(norm, L.norm) and all(torch.equal(a, b) for a, b in zip(first, L.clipped))
    before = [g.clone() for g in grads]
    alone = torch.zeros((), device="cuda")
    twice = grads + grads[:1]                            # the norm alone may read a tensor twice
    sizes, types = [*L.sizes, L.sizes[0]], [*L.dtypes, L.dtypes[0]]
    ws = torch.empty(B.rgnn_clip_workspace_bytes(sizes), dtype=torch.uint8, device="cuda")
    B.rgnn_clip_grad_norm(grads, None, L.sizes, L.dtypes, float("nan"), alone, ws)
    assert torch.equal(alone, norm) and all(torch.equal(a, b) for a, b in zip(before, grads))
    B.rgnn_clip_grad_norm(twice, None, sizes, types, 0.0, alone, ws)
    want = math.sqrt(sum(float(g.double().pow(2).sum()) for g in twice))
    assert abs(float(alone) - want) <= want * 1.01 * U


def test_a_tensor_past_32_bits():
    import torch
    from paper_2412_04747_amd.harness import GradClip
    n = (1 << 31) + 4111
    print(f"clip case of {n} elements", flush=True)
    g = [torch.ones(n, device="cuda", dtype=torch.bfloat16)]
    g[0][-1] = 3.0
    want = math.sqrt(n - 1 + 9)
    L = GradClip(g)
    L.clip(g, want / 2)
    assert abs(float(L.norm) - want) <= want * 1.01 * U
    assert float(g[0][0]) == 0.5 and float(g[0][n // 2]) == 0.5 and float(g[0][-1]) == 1.5 and bool((g[0][-10000:-1] == 0.5).all())
