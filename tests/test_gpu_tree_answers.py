"""What PagedStack.verify answers beside the rows that stay: pages that the free list lacked."""
import numpy as np
import pytest
import torch

from paper_2601_12904_amd import stack as S
from tests.test_gpu_paged import i32, make_ctx
from tests.test_gpu_tree import forest
from tests.test_gpu_tree_stack import make_layers

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_pages,lacks", [(12, 0), (7, 0), (6, 1), (3, 4)])
def test_a_step_whose_free_list_is_too_short_says_so(n_pages, lacks):
    """Two requests of 30 and 20 rows in pages of 8: seven pages.  What verify() gives back afterwards does not hide that the list had fewer."""
    hidden, vocab, page = 256, 256, 8
    gen = torch.Generator(device="cuda").manual_seed(3)
    layers, _ = make_layers(1, hidden, 384, 8, 2, 128, gen, True)
    ctx = make_ctx((8, 2, 128, "bf16"), tokens=64)
    stack, head = S.PagedStack(ctx, layers, hidden, 384), S.Head(ctx, S.random_head(hidden, vocab, gen, std=0.1))
    cache = S.PagedCache(1, 2, n_pages, page, 8, 2, 128)
    rng = np.random.default_rng(1)
    parents = np.concatenate([forest(rng, 30, "tree"), forest(rng, 20, "tree")])
    h = torch.randn((50, hidden), generator=gen, device="cuda").bfloat16()
    got = stack.verify(h, i32(parents), i32(np.full(50, -1)), i32([30, 20]), 30, cache, head)     # (no draft agrees: row 0 of each stays)
    assert got["free_end"].tolist() == [7] and max(0, got["free_end"].item() - n_pages) == lacks
    assert got["kept"].tolist() == [1, 1] and cache.cached_len.tolist() == [1, 1]
    # request 0 took the first four pages of the list, request 1 the next three; each keeps its first one
    stays = [p for p in (0, 4) if p < n_pages]
    assert cache.free_start.tolist() == [len(stays)]
    assert sorted(cache.free_pages[len(stays):].tolist() + stays) == list(range(n_pages))
    ctx.close()
