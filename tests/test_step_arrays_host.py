"""Arrays that a head or a step over a paged cache would read past their end, or as what they are not, are refused before anything is launched."""
import pytest
import torch

from paper_2601_12904_amd import binding as B
from paper_2601_12904_amd import stack as S

BF, I32 = torch.bfloat16, torch.int32


@pytest.fixture
def ctx():
    c = B.Context(4, 2, 128, B.FR_BF16, 1e4, max_tokens=64, max_chunks=1, max_question_tokens=1)
    yield c
    c.close()


def weights(vocab=128, hidden=64, dtype=BF, g=None):
    return S.HeadWeights(torch.ones(hidden if g is None else g, dtype=dtype), torch.ones(vocab, hidden, dtype=dtype))


def on(w, device):
    return S.HeadWeights(w.g.to(device), w.w.to(device))


@pytest.mark.parametrize("h,tokens,match", [
    ((6, 64), 5, "tokens has shape"), ((6, 64), 7, "tokens has shape"), ((6, 64), (6, 1), "tokens has shape"), ((6, 64), 0, "tokens has shape"),
    ((6, 32), 6, "h has shape"), ((6, 128), None, "h has shape"), ((64,), None, "h has shape"), ((1, 6, 64), None, "h has shape")])
def test_rows_and_tokens_of_other_sizes_are_refused(ctx, h, tokens, match):
    tokens = None if tokens is None else torch.zeros(tokens, dtype=I32)
    with pytest.raises(ValueError, match=match):
        S.Head(ctx, weights()).logprobs(torch.zeros(h, dtype=BF), tokens)


def test_rows_and_weights_of_other_types_are_refused(ctx):
    with pytest.raises(ValueError, match="h is of torch.float32"):
        S.Head(ctx, weights()).logprobs(torch.zeros(6, 64))
    for dtype in (torch.float32, torch.float16):
        with pytest.raises(ValueError, match="weights are of"):
            S.Head(ctx, weights(dtype=dtype)).logprobs(torch.zeros((6, 64), dtype=BF))


def test_a_norm_of_another_width_is_refused(ctx):
    for g in (32, 128):
        with pytest.raises(ValueError, match="g has shape"):
            S.Head(ctx, weights(g=g))


def test_arrays_that_are_not_on_the_gpu_are_refused(ctx):
    """(The library takes addresses: one of the host's would be read by a kernel.)"""
    h = torch.zeros((6, 64), dtype=BF)
    with pytest.raises(ValueError, match="h: on cpu"):
        S.Head(ctx, weights()).logprobs(h)
    with pytest.raises(ValueError, match="tokens: on cpu, h on meta"):
        S.Head(ctx, on(weights(), "meta")).logprobs(h.to("meta"), torch.zeros(6, dtype=I32))
    with pytest.raises(ValueError, match="weights: on cpu, h on meta"):
        S.Head(ctx, weights()).logprobs(h.to("meta"))
