"""Layers that PagedStack cannot run are refused when it is made, not in the middle of a step."""
import pytest

from paper_2601_12904_amd import binding as B
from paper_2601_12904_amd import stack as S


def make(Hq, Hkv, d, layout):
    ctx = B.Context(Hq, Hkv, d, B.FR_BF16, 1e4, max_tokens=64, max_chunks=1, max_question_tokens=1, rope_layout=layout)
    try:
        return S.PagedStack(ctx, [], 256, 256)
    finally:
        ctx.close()


@pytest.mark.parametrize("Hq,Hkv,layout", [(6, 3, B.FR_ROPE_INTERLEAVED), (6, 3, B.FR_ROPE_HALF), (7, 1, B.FR_ROPE_HALF), (4, 1, B.FR_ROPE_INTERLEAVED)])
def test_parts_that_are_no_multiple_of_128_features(Hq, Hkv, layout):
    with pytest.raises(ValueError, match="128"):
        make(Hq, Hkv, 64, layout)


@pytest.mark.parametrize("Hq,Hkv,d,layout", [(6, 2, 64, B.FR_ROPE_HALF), (7, 1, 128, B.FR_ROPE_INTERLEAVED), (7, 1, 128, B.FR_ROPE_HALF)])
def test_others_are_taken(Hq, Hkv, d, layout):
    assert make(Hq, Hkv, d, layout).fused_rope == (d == 128 and layout == B.FR_ROPE_INTERLEAVED)
