"""Arguments that rows in 8 bits, the junction of a block and the feed-forward backward from held rows refuse: all checks are made on the host before any
device call (no GPU needed)."""
import os

import pytest

from paper_2412_04747_amd import binding as B

EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 5
A = [4096 * (1 << 16) * k for k in range(1, 30)]          # addresses 256 MB apart; never read


@pytest.fixture(autouse=True, scope="module")
def built():
    if not os.path.exists(B.LIB_PATH):
        from paper_2412_04747_amd import build
        build.build()


def refused(status, word, f, *args):
    with pytest.raises(B.RgnnError) as e:
        f(*args)
    assert e.value.status == status and word in str(e.value), e.value


@pytest.mark.parametrize("change,status,word", [(dict(rows=-1), EINVAL, "rows"), (dict(rows=1 << 31), EUNSUPPORTED, "rows"), (dict(width=0), EINVAL, "width"),
                                                (dict(width=8193), EUNSUPPORTED, "width"), (dict(dtype=2), EINVAL, "dtype")])
def test_rows8_descriptor(change, status, word):
    d = B.make_rows8_desc(**dict(dict(rows=10, width=64), **change))
    refused(status, word, B.rgnn_rows8_pack, d, A[0], B.rows8(A[1], A[2]))
    refused(status, word, B.rgnn_rows8_unpack, d, B.rows8(A[1], A[2]), A[0])


def test_rows8_pointers():
    d = B.make_rows8_desc(10, 64)
    for f in (lambda x, r: B.rgnn_rows8_pack(d, x, r), lambda x, r: B.rgnn_rows8_unpack(d, r, x)):
        refused(EINVAL, "NULL", f, None, B.rows8(A[1], A[2]))
        refused(EINVAL, "NULL", f, A[0], None)
        refused(EINVAL, "NULL", f, A[0], B.rows8(None, A[2]))
        refused(EINVAL, "NULL", f, A[0], B.rows8(A[1], None))
        refused(EINVAL, "aligned", f, A[0] + 4, B.rows8(A[1], A[2]))
        refused(EINVAL, "aligned", f, A[0], B.rows8(A[1] + 8, A[2]))
        refused(EINVAL, "overlap", f, A[0], B.rows8(A[0] + 256, A[2]))
        refused(EINVAL, "overlap", f, A[0], B.rows8(A[1], A[0] + 1))
        refused(EINVAL, "overlap", f, A[0], B.rows8(A[1], A[1] + 639))
    assert B.rgnn_rows8_pack(B.make_rows8_desc(0, 64), None, None) is None


# ---- junction

def desc(**k):
    return B.make_block_norm_desc(**dict(dict(rows=10, width=64, types=2), **k))


def params(**k):
    return B.block_norm_params(**dict(dict(row_types=A[0], w_after=A[1], gate=A[2], scale=A[3], w_before=A[4]), **k))


a, s, total, out, dy, ds, da, dstream, ws = A[5:14]
grads = lambda **k: B.block_norm_grads(**dict(dict(w_after=A[14], gate=A[15], scale=A[16], w_before=A[17]), **k))
a8, s8 = (lambda **k: B.rows8(**dict(dict(codes=A[18], scales=A[19]), **k))), (lambda **k: B.rows8(**dict(dict(codes=A[20], scales=A[21]), **k)))


@pytest.mark.parametrize("change,status,word", [
    (dict(rows=-1), EINVAL, "rows"), (dict(rows=1 << 31), EUNSUPPORTED, "rows"), (dict(width=0), EINVAL, "width"), (dict(width=8193), EUNSUPPORTED, "width"),
    (dict(a_dtype=2), EINVAL, "dtype"), (dict(sum_dtype=-1), EINVAL, "dtype"), (dict(out_dtype=7), EINVAL, "dtype"), (dict(types=0), EINVAL, "types"),
    (dict(types=-3), EINVAL, "types"), (dict(types=54), EUNSUPPORTED, "types"), (dict(types=2, width=2037), EUNSUPPORTED, "types"), (dict(eps=-1e-6), EINVAL, "eps"),
    (dict(eps=float("nan")), EINVAL, "eps"), (dict(eps=float("inf")), EINVAL, "eps"), (dict(flags=1), EINVAL, "flags")])
def test_block_norm_descriptor(change, status, word):
    d = desc(**change)
    refused(status, word, B.rgnn_block_norm_workspace_bytes, d)
    refused(status, word, B.rgnn_block_norm_fwd, d, params(), a, s, total, out)
    refused(status, word, B.rgnn_block_norm_bwd, d, params(), a, s, None, None, dy, ds, da, dstream, grads(), ws)


def test_block_norm_sizes_that_are_taken():
    for types, width in ((1, 8192), (53, 64), (2, 2036), (4, 1012), (315, 1), (29, 128)):
        assert B.rgnn_block_norm_workspace_bytes(desc(types=types, width=width, rows=100000)) > 0


def test_block_norm_forward_pointers():
    f, d = B.rgnn_block_norm_fwd, desc()
    refused(EINVAL, "params", f, d, None, a, s, total, out)
    refused(EINVAL, "row_types", f, d, params(row_types=None), a, s, total, out)
    refused(EINVAL, "NULL", f, d, params(), None, s, total, out)
    refused(EINVAL, "NULL", f, d, params(), a, None, total, out)
    refused(EINVAL, "w_before", f, d, params(w_before=None), a, s, total, out)
    refused(EINVAL, "w_before", f, d, params(), a, s, total, None)
    refused(EINVAL, "no result", f, d, params(w_before=None), a, s, None, None)
    refused(EINVAL, "together", f, d, params(), a, s, total, out, a8())
    refused(EINVAL, "together", f, d, params(), a, s, total, out, None, s8())
    refused(EINVAL, "NULL", f, d, params(), a, s, total, out, a8(), s8(scales=None))
    for k in ("row_types", "w_after", "gate", "scale", "w_before"):
        at = getattr(params(), k)
        refused(EINVAL, "aligned", f, d, params(**{k: at + 4}), a, s, total, out)
        refused(EINVAL, "parameter", f, d, params(), a, s, at, out)
        refused(EINVAL, "parameter", f, d, params(), a, s, total, out, a8(), s8(codes=at))
    refused(EINVAL, "aligned", f, d, params(), a + 8, s, total, out)
    refused(EINVAL, "aligned", f, d, params(), a, s, total, out + 2)
    refused(EINVAL, "aligned", f, d, params(), a, s, total, out, a8(codes=A[18] + 1), s8())
    refused(EINVAL, "buffer of", f, d, params(), a, s, a + 256, out)
    refused(EINVAL, "buffer of", f, d, params(), a, s, total, s - 256)
    refused(EINVAL, "buffer of", f, desc(out_dtype=B.RGNN_BF16), params(), a, s, total, s)          # the same place in another type
    refused(EINVAL, "overlap", f, d, params(), a, s, total, total)
    refused(EINVAL, "a8 or s8", f, d, params(), a, s, total, out, a8(codes=a), s8())
    refused(EINVAL, "a8 or s8", f, d, params(), a, s, total, out, a8(), s8(scales=out + 3))
    refused(EINVAL, "codes and scales", f, d, params(), a, s, total, out, a8(), s8(codes=A[18]))
    refused(EINVAL, "codes and scales", f, d, params(), a, s, total, out, a8(scales=A[18] + 100), s8())
    assert f(desc(rows=0), params(row_types=None), None, None, None, None) is None


def test_block_norm_backward_pointers():
    f, d = B.rgnn_block_norm_bwd, desc()
    n = (None, None)
    refused(EINVAL, "params", f, d, None, a, s, *n, dy, ds, da, dstream, grads(), ws)
    refused(EINVAL, "row_types", f, d, params(row_types=None), a, s, *n, dy, ds, da, dstream, grads(), ws)
    refused(EWORKSPACE, "workspace", f, d, params(), a, s, *n, dy, ds, da, dstream, grads(), None)
    for k in ("w_after", "gate", "scale", "w_before"):
        refused(EINVAL, "not given", f, d, params(**{k: None}), a, s, *n, dy, ds, da, dstream, grads(), ws)
        refused(EINVAL, "aligned", f, d, params(), a, s, *n, dy, ds, da, dstream, grads(**{k: A[15] + 4}), ws)
        refused(EINVAL, "overlap", f, d, params(), a, s, *n, dy, ds, da, dstream, grads(**{k: dy + 512}), ws)
        refused(EINVAL, "overlap", f, d, params(), a, s, *n, dy, ds, da, dstream, grads(**{k: ws}), ws)
        refused(EINVAL, "parameter", f, d, params(), a, s, *n, dy, ds, da, dstream, grads(**{k: getattr(params(), k)}), ws)
    refused(EINVAL, "a and s", f, d, params(), None, s, *n, dy, ds, da, dstream, grads(), ws)
    refused(EINVAL, "a and s", f, d, params(), a, None, *n, dy, ds, da, dstream, grads(), ws)
    refused(EINVAL, "a and s", f, d, params(), a, s, a8(), s8(), dy, ds, da, dstream, grads(), ws)
    refused(EINVAL, "together", f, d, params(), None, None, a8(), None, dy, ds, da, dstream, grads(), ws)
    refused(EINVAL, "NULL", f, d, params(), None, None, a8(), s8(codes=None), dy, ds, da, dstream, grads(), ws)
    refused(EINVAL, "both NULL", f, d, params(), a, s, *n, None, None, da, dstream, grads(), ws)
    refused(EINVAL, "w_before", f, d, params(w_before=None), a, s, *n, dy, ds, da, dstream, grads(w_before=None), ws)
    refused(EINVAL, "aligned", f, d, params(), a, s, *n, dy + 4, ds, da, dstream, grads(), ws)
    refused(EINVAL, "aligned", f, d, params(), a, s, *n, dy, ds, da, dstream, grads(), ws + 4)
    refused(EINVAL, "buffer of", f, d, params(), a, s, *n, dy, ds, a, dstream, grads(), ws)
    refused(EINVAL, "buffer of", f, d, params(), a, s, *n, dy, ds, da, s, grads(), ws)
    refused(EINVAL, "buffer of", f, d, params(), a, s, *n, dy, ds, dy + 256, dstream, grads(), ws)
    refused(EINVAL, "buffer of", f, d, params(), None, None, a8(), s8(), dy, ds, da, A[19], grads(), ws)
    refused(EINVAL, "dA and dS", f, d, params(), a, s, *n, dy, ds, da, da, grads(), ws)
    refused(EINVAL, "overlap", f, d, params(), a, s, *n, dy, ds, da, dstream, grads(), s + 256)
    refused(EINVAL, "overlap", f, d, params(), a, s, *n, dy, ds, da, dstream, grads(scale=A[15]), ws)


# ---- feed-forward block from held rows

def test_ffn_rows8():
    f = B.rgnn_ffn_bwd_rows8
    X8 = lambda **k: B.rows8(**dict(dict(codes=A[0], scales=A[1]), **k))
    w = (A[2], A[3], A[4])
    g = (A[7], A[8], A[9])
    d = B.make_ffn_desc(rows=10, width=64, hidden=100)
    refused(EUNSUPPORTED, "width", f, B.make_ffn_desc(rows=10, width=48, hidden=100), X8(), *w, A[5], A[6], *g, A[10])
    refused(EINVAL, "X8", f, d, None, *w, A[5], A[6], *g, A[10])
    refused(EINVAL, "X ", f, d, X8(codes=None), *w, A[5], A[6], *g, A[10])
    refused(EINVAL, "X ", f, d, X8(scales=None), *w, A[5], A[6], *g, A[10])
    refused(EINVAL, "aligned", f, d, X8(codes=A[0] + 8), *w, A[5], A[6], *g, A[10])
    refused(EINVAL, "overlaps", f, d, X8(), *w, A[5], A[0] + 624, *g, A[10])
    refused(EINVAL, "scales", f, d, X8(), *w, A[5], A[1], *g, A[10])
    refused(EINVAL, "scales", f, d, X8(), *w, A[5], A[6], *g, A[1] - 256)
    refused(EINVAL, "weight", f, d, X8(), None, A[3], A[4], A[5], A[6], *g, A[10])
    refused(EINVAL, "together", f, d, X8(), *w, A[5], A[6], A[7], None, A[9], A[10])
    refused(EWORKSPACE, "workspace", f, d, X8(), *w, A[5], A[6], *g, None)


def test_declared_argument_counts():
    """ctypes passes what goes past a function's declared arguments as 32-bit numbers."""
    import re
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(os.path.dirname(B.HERE), "include", "rgnn.h")).read(), flags=re.S)
    for name, args in re.findall(r"\b(rgnn_\w+)\s*\(([^;]*?)\)\s*;", header, re.S):
        if name in B._ROW_OPS:
            assert len(args.split(",")) == len(B._ROW_OPS[name]), name


def test_block_norm_of_every_drawn_workload():
    """Up to 8 types of up to 1024 columns, as the workloads draw them, and what lies between."""
    import random
    from perf import more_operators as M
    code = dict(f32=B.RGNN_F32, bf16=B.RGNN_BF16)
    rng = random.Random(5)
    wide = 0
    for c in [*M.listed(), *(M.draw(rng) for _ in range(6000))]:
        if c["op"] == "block":
            wide += c["types"] > 1 and c["types"] * (c["width"] + 12) > 4096
            d = desc(rows=c["rows"], width=c["width"], types=c["types"], a_dtype=code[c["a"]], sum_dtype=code[c["total"]], out_dtype=code[c["out"]])
            assert B.rgnn_block_norm_workspace_bytes(d) > 0, c
    assert wide > 5
    for types, width in ((8, 1024), (8, 512), (5, 1000), (4, 1024), (2, 1024), (30, 128), (32, 278), (16, 552)):
        for t in code.values():
            assert B.rgnn_block_norm_workspace_bytes(desc(types=types, width=width, rows=100000, a_dtype=t, sum_dtype=t, out_dtype=t)) > 0
    for types, width in ((9, 1024), (33, 200), (32, 279), (4, 1025)):
        refused(EUNSUPPORTED, "types", B.rgnn_block_norm_workspace_bytes, desc(types=types, width=width))
