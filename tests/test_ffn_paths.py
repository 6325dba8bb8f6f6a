"""Which calls of the feed-forward block have their weights laid out first, told by the workspace they ask for (no GPU needed): laid-out weights are
three sections of 32 hidden values' rows in bf16 planes, three of fp32."""
import pytest

from paper_2412_04747_amd import binding as B


def _laid_out(rows, width, hidden, dtype, backward=False):
    d = B.make_ffn_desc(rows, width, hidden, B.RGNN_BF16 if dtype == "bf16" else B.RGNN_F32)
    weights = (5 if backward else 3) * width * 32 * ((hidden + 31) // 32) * 2 * (1 if dtype == "bf16" else 3)
    got = B.rgnn_ffn_workspace_bytes(d)[backward]
    return (weights + 255) // 256 * 256 == got if not backward else got >= weights


# Rows of many chunks, which a workgroup that lays out its own weights would take one after the other.
@pytest.mark.parametrize("rows,width,hidden,dtype", [(32768, 32, 512, "bf16"), (32768, 32, 512, "f32"), (20000, 32, 16384, "bf16"), (8000, 32, 128, "bf16"),
                                                     (16000, 32, 96, "f32"), (3000, 32, 2048, "bf16"), (8000, 128, 128, "f32"), (1000, 128, 64, "f32"),
                                                     (1000, 64, 128, "bf16"), (1 << 20, 32, 20, "bf16")])
def test_many_chunks_in_turn_are_laid_out(rows, width, hidden, dtype):
    assert _laid_out(rows, width, hidden, dtype)


# Few rows, or a chunk or two: launches are the time.
@pytest.mark.parametrize("rows,width,hidden,dtype", [(1, 128, 64, "bf16"), (4, 128, 64, "f32"), (300, 32, 100, "bf16"), (1000, 32, 86, "f32"), (1000, 32, 2048, "bf16"),
                                                     (4000, 128, 512, "f32"), (32768, 32, 64, "bf16"), (32768, 32, 40, "f32"), (32768, 128, 32, "f32")])
def test_few_rows_or_chunks_are_not(rows, width, hidden, dtype):
    assert not _laid_out(rows, width, hidden, dtype)


def test_rows_decide_once():
    """With more rows a call does not go back to the kernels for few (one row and up to four in fp32 aside)."""
    for width in (32, 64, 128):
        for hidden in (1, 32, 33, 64, 65, 97, 256, 2048, 16384):
            for dtype in ("bf16", "f32"):
                laid = [_laid_out(rows, width, hidden, dtype) for rows in (5, 64, 200, 700, 1500, 3000, 5000, 8192, 8193, 20000, 32768, 32769, 100000)]
                assert laid == sorted(laid) and laid[-1], (width, hidden, dtype)
