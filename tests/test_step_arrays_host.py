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


def step(ctx, **change):
    from types import SimpleNamespace
    zeros = lambda n: torch.zeros(n, dtype=I32)
    call = dict(h=torch.zeros((6, 64), dtype=BF), parents=zeros(6), tokens=zeros(6), new_len=zeros(2), max_new=3, cache=SimpleNamespace(n_requests=2, k=[], v=[]), head=S.Head(ctx, weights()))
    return dict(call, **change)


@pytest.mark.parametrize("change,match", [
    (dict(h=torch.zeros((6, 32), dtype=BF)), "h has shape"), (dict(h=torch.zeros((6, 64, 1), dtype=BF)), "h has shape"), (dict(h=torch.zeros(6, 64)), "h is of torch.float32"),
    (dict(new_len=torch.zeros(2)), "int32"), (dict(new_len=torch.zeros(1, dtype=I32)), "new_len has shape"), (dict(new_len=torch.zeros(2, dtype=I32, device="meta")), "new_len: on meta"),
    (dict(), "h: on cpu")])
def test_steps_that_read_other_arrays_are_refused(ctx, change, match):
    call = step(ctx, **change)
    stack = S.PagedStack(ctx, [], 64, 64)
    with pytest.raises(ValueError, match=match):
        stack.verify(**call)
    with pytest.raises(ValueError, match=match):
        stack.forward(call["h"], call["new_len"], 3, call["cache"])


@pytest.mark.parametrize("name", ["parents", "tokens", "given"])
def test_drafts_of_another_device_are_refused(ctx, name):
    with pytest.raises(ValueError, match=f"{name}: on meta"):
        S.PagedStack(ctx, [], 64, 64).verify(**step(ctx, **{name: torch.zeros(2 if name == "given" else 6, dtype=I32, device="meta")}))


def test_a_head_of_another_width_is_refused(ctx):
    with pytest.raises(ValueError, match="128 features"):
        S.PagedStack(ctx, [], 64, 64).verify(**step(ctx, head=S.Head(ctx, weights(hidden=128))))


def test_more_layers_than_rows_can_be_kept_in_are_refused_before_the_step(ctx):
    """(Behind the step, when fr_tree_keep refuses them, all of its work is lost.)"""
    from types import SimpleNamespace
    pages = [None] * (B.FR_TREE_MAX_LAYERS + 1)
    with pytest.raises(ValueError, match="129 layers"):
        S.PagedStack(ctx, [], 64, 64).verify(**step(ctx, cache=SimpleNamespace(n_requests=2, k=pages, v=pages)))
