"""Arguments that the row operators and the gradient clipping refuse: all checks are made on the host before any device call (no GPU needed)."""
import ctypes as C
import os

import pytest

from paper_2412_04747_amd import binding as B

EINVAL, EUNSUPPORTED, EWORKSPACE = 1, 2, 5
A = [4096 * (1 << 16) * k for k in range(1, 16)]          # addresses 256 MB apart; never read


@pytest.fixture(autouse=True, scope="module")
def built():
    if not os.path.exists(B.LIB_PATH):
        from paper_2412_04747_amd import build
        build.build()


def refused(status, word, f, *args):
    with pytest.raises(B.RgnnError) as e:
        f(*args)
    assert e.value.status == status and word in str(e.value), e.value


# ---- norm

def norm(**k):
    d = dict(rows=10, width=64)
    d.update(k)
    return B.make_norm_desc(**d)


@pytest.mark.parametrize("change,status,word", [
    (dict(rows=-1), EINVAL, "rows"), (dict(rows=1 << 31), EUNSUPPORTED, "rows"), (dict(width=0), EINVAL, "width"),
    (dict(width=8193), EUNSUPPORTED, "width"), (dict(x_dtype=2), EINVAL, "dtype"), (dict(sum_dtype=-1), EINVAL, "dtype"),
    (dict(out_dtype=7), EINVAL, "dtype"), (dict(eps=-1e-6), EINVAL, "eps"), (dict(eps=float("nan")), EINVAL, "eps"),
    (dict(eps=float("inf")), EINVAL, "eps"), (dict(flags=1), EINVAL, "flags")])
def test_norm_descriptor(change, status, word):
    d = norm(**change)
    refused(status, word, B.rgnn_norm_workspace_bytes, d)
    refused(status, word, B.rgnn_norm_fwd, d, A[0], None, A[1], None, A[2])
    refused(status, word, B.rgnn_norm_bwd, d, A[0], A[1], A[2], None, A[3], None, A[4], A[5])


def test_norm_pointers():
    d = norm()
    refused(EINVAL, "weight", B.rgnn_norm_fwd, d, A[0], None, None, None, A[2])
    refused(EINVAL, "NULL", B.rgnn_norm_fwd, d, None, None, A[1], None, A[2])
    refused(EINVAL, "NULL", B.rgnn_norm_fwd, d, A[0], None, A[1], None, None)
    refused(EINVAL, "aligned", B.rgnn_norm_fwd, d, A[0] + 4, None, A[1], None, A[2])
    refused(EINVAL, "aligned", B.rgnn_norm_fwd, d, A[0], None, A[1], A[3] + 8, A[2])
    refused(EINVAL, "overlaps", B.rgnn_norm_fwd, d, A[0], None, A[1], None, A[0] + 256)          # shifted by a row
    refused(EINVAL, "overlaps", B.rgnn_norm_fwd, d, A[0], A[2], A[1], A[2] - 256, A[3])
    refused(EINVAL, "overlaps", B.rgnn_norm_fwd, d, A[0], None, A[1], None, A[1])
    refused(EINVAL, "overlap", B.rgnn_norm_fwd, d, A[0], None, A[1], A[2], A[2])
    # the same place in another type is a shifted overlap
    refused(EINVAL, "overlaps", B.rgnn_norm_fwd, norm(out_dtype=B.RGNN_BF16), A[0], None, A[1], None, A[0])
    bwd = B.rgnn_norm_bwd
    refused(EINVAL, "weight", bwd, d, A[0], None, A[2], None, A[3], None, A[4], A[5])
    refused(EINVAL, "NULL", bwd, d, None, A[1], A[2], None, A[3], None, A[4], A[5])
    refused(EINVAL, "NULL", bwd, d, A[0], A[1], None, None, A[3], None, A[4], A[5])
    refused(EWORKSPACE, "workspace", bwd, d, A[0], A[1], A[2], None, A[3], None, A[4], None)
    refused(EINVAL, "overlaps", bwd, d, A[0], A[1], A[2], None, A[0], None, A[4], A[5])           # dX over sum
    refused(EINVAL, "overlaps", bwd, d, A[0], A[1], A[2], None, A[3], None, A[4], A[3] + 256)     # workspace over dX
    refused(EINVAL, "overlap", bwd, d, A[0], A[1], A[2], None, A[3], A[3], A[4], A[5])
    refused(EINVAL, "dWeight", bwd, d, A[0], A[1], A[2], None, A[3], None, A[2], A[5])
    refused(EINVAL, "aligned", bwd, d, A[0], A[1], A[2], None, A[3], None, A[4], A[5] + 4)
    refused(EINVAL, "workspace", bwd, d, A[0], A[1], A[2], None, A[3], None, A[4], A[0] + 256)    # workspace over sum
    refused(EINVAL, "workspace", bwd, d, A[0], A[1], A[2], None, A[3], None, A[4], A[4])          # workspace over dWeight


# ---- feed-forward block

def ffn(**k):
    d = dict(rows=10, width=64, hidden=100)
    d.update(k)
    return B.make_ffn_desc(**d)


@pytest.mark.parametrize("change,status,word", [
    (dict(rows=-1), EINVAL, "rows"), (dict(rows=1 << 31), EUNSUPPORTED, "rows"), (dict(width=48), EUNSUPPORTED, "width"),
    (dict(width=256), EUNSUPPORTED, "width"), (dict(hidden=0), EINVAL, "hidden"), (dict(hidden=16385), EUNSUPPORTED, "hidden"),
    (dict(dtype=2), EINVAL, "dtype"), (dict(activation=0), EINVAL, "activation"), (dict(activation=3), EINVAL, "activation"),
    (dict(flags=64), EINVAL, "flags")])
def test_ffn_descriptor(change, status, word):
    d = ffn(**change)
    refused(status, word, B.rgnn_ffn_workspace_bytes, d)
    refused(status, word, B.rgnn_ffn_fwd, d, *A[:6])
    refused(status, word, B.rgnn_ffn_bwd, d, *A[:10])


def test_ffn_pointers():
    d = ffn()
    for i in range(5):
        refused(EINVAL, "NULL", B.rgnn_ffn_fwd, d, *[None if k == i else a for k, a in enumerate(A[:6])])
    refused(EWORKSPACE, "workspace", B.rgnn_ffn_fwd, d, *A[:5], None)
    refused(EINVAL, "aligned", B.rgnn_ffn_fwd, d, A[0], A[1] + 4, *A[2:6])
    refused(EINVAL, "overlaps", B.rgnn_ffn_fwd, d, *A[:4], A[0], A[5])                   # out over X
    refused(EINVAL, "overlaps", B.rgnn_ffn_fwd, d, *A[:4], A[4], A[3] - 256)             # workspace over Wd
    refused(EINVAL, "overlap", B.rgnn_ffn_fwd, d, *A[:4], A[4], A[4])
    for i in range(5):
        refused(EINVAL, "NULL", B.rgnn_ffn_bwd, d, *[None if k == i else a for k, a in enumerate(A[:10])])
    refused(EWORKSPACE, "workspace", B.rgnn_ffn_bwd, d, *A[:9], None)
    refused(EINVAL, "together", B.rgnn_ffn_bwd, d, *A[:6], None, *A[7:10])
    refused(EINVAL, "overlaps", B.rgnn_ffn_bwd, d, *A[:5], A[4], *A[6:10])               # dX over dOut
    refused(EINVAL, "overlap", B.rgnn_ffn_bwd, d, *A[:7], A[6], *A[8:10])                # dWu over dWg


# ---- clipping

def clip(grads=(A[0], A[1]), clipped=(A[2], A[3]), sizes=(100, 100), dtypes=(0, 0), max_norm=1.0, norm=A[4], ws=A[5]):
    B.rgnn_clip_grad_norm(list(grads), None if clipped is None else list(clipped), list(sizes), list(dtypes), max_norm, norm, ws)


@pytest.mark.parametrize("change,status,word", [
    (dict(sizes=(100, -1)), EINVAL, "size"), (dict(sizes=(100, (1 << 40) + 1)), EINVAL, "size"), (dict(dtypes=(0, 2)), EINVAL, "dtype"),
    (dict(max_norm=-1.0), EINVAL, "max_norm"), (dict(max_norm=float("nan")), EINVAL, "max_norm"), (dict(norm=None), EINVAL, "norm"),
    (dict(ws=None), EWORKSPACE, "workspace"), (dict(ws=A[5] + 4), EINVAL, "aligned"), (dict(norm=A[4] + 2), EINVAL, "aligned"),
    (dict(grads=(A[0], None)), EINVAL, "NULL"), (dict(clipped=(None, A[3])), EINVAL, "NULL"),
    (dict(grads=(A[0], A[1] + 2)), EINVAL, "aligned"), (dict(grads=(A[0], A[1] + 1), dtypes=(0, 1)), EINVAL, "aligned"),
    (dict(clipped=(A[2], A[2])), EINVAL, "overlaps"),                                    # two results in one place
    (dict(grads=(A[0], A[0]), clipped=(A[0], A[0])), EINVAL, "overlaps"),                # in place, given twice
    (dict(clipped=(A[0] + 4, A[3])), EINVAL, "overlaps"),                                # shifted by an element
    (dict(clipped=(A[1], A[0])), EINVAL, "overlaps"),                                    # each over the other's gradient
    (dict(clipped=None, norm=A[1] + 40), EINVAL, "overlaps"),                            # the norm into a gradient
    (dict(ws=A[1] + 16), EINVAL, "overlaps"), (dict(ws=A[4]), EINVAL, "overlaps"),       # the workspace into a gradient, or the norm
    (dict(grads=(A[0], A[0] + 200), clipped=(A[0], A[0] + 200), dtypes=(0, 1)), EINVAL, "overlaps")])
def test_clip_refusals(change, status, word):
    refused(status, word, lambda: clip(**change))


def test_clip_raw_null_arrays():
    lib = B.lib()
    n = C.c_size_t()
    assert lib.rgnn_clip_workspace_bytes(C.c_int64(-1), None, C.byref(n)) == EINVAL
    assert lib.rgnn_clip_workspace_bytes(C.c_int64(1), None, C.byref(n)) == EINVAL
    assert lib.rgnn_clip_workspace_bytes(C.c_int64(0), None, C.byref(n)) == 0 and n.value > 0
    one = (C.c_int64 * 1)(5)
    assert lib.rgnn_clip_grad_norm(C.c_int64(1), None, None, one, None, C.c_float(1), C.c_void_p(A[0]), C.c_void_p(A[1]), None) == EINVAL


def test_no_rows_enqueue_nothing():
    """Without rows the row tensors may be NULL and no launch is made (none could be here)."""
    B.rgnn_norm_fwd(norm(rows=0), None, None, A[0], None, None)
    B.rgnn_norm_bwd(norm(rows=0), None, A[0], None, None, None, None, None, None)
    B.rgnn_norm_bwd(norm(rows=0, flags=B.RGNN_FLAG_ACCUMULATE), None, A[0], None, None, None, None, A[1], A[2])
    B.rgnn_ffn_fwd(ffn(rows=0), None, A[0], A[1], A[2], None, None)
    B.rgnn_ffn_bwd(ffn(rows=0), None, A[0], A[1], A[2], None, None, None, None, None, A[3])
