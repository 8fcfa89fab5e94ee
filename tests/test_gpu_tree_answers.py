"""What PagedStack.verify answers beside the rows that stay: choices, log probabilities and entropies of its own logits, and pages that the free list lacked."""
import numpy as np
import pytest
import torch

from paper_2601_12904_amd import stack as S
from tests import test_gpu_logprobs as lp
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


@pytest.mark.parametrize("Hq,Hkv,d,qk_norm", [(8, 2, 128, False), (8, 4, 64, True)])
def test_answers_are_those_of_the_steps_logits(Hq, Hkv, d, qk_norm):
    """The logits of the rows that a step left, projected once more by the library's own calls, and the 64-bit oracle on those logits: to the bounds of fp32, not to those of a layer in bf16."""
    hidden, vocab = 256, 640
    gen = torch.Generator(device="cuda").manual_seed(4)
    layers, _ = make_layers(2, hidden, 384, Hq, Hkv, d, gen, qk_norm)
    ctx = make_ctx((Hq, Hkv, d, "bf16"), tokens=64)
    headw = S.random_head(hidden, vocab, gen, std=0.2)
    stack, head = S.PagedStack(ctx, layers, hidden, 384), S.Head(ctx, headw)
    cache = S.PagedCache(2, 2, 20, 8, 8, Hkv, d)
    rng = np.random.default_rng(2)
    for new in ([21, 13], [1, 30]):
        T = sum(new)
        parents, tokens = np.concatenate([forest(rng, n, "tree") for n in new]), rng.integers(0, vocab, T)
        h = torch.randn((T, hidden), generator=gen, device="cuda").bfloat16()
        got = stack.verify(h, i32(parents), i32(tokens), i32(new), max(new), cache, head)
        x, logits = torch.empty_like(h), torch.empty((T, vocab), dtype=torch.bfloat16, device="cuda")
        ctx.fr_rmsnorm(h, headw.g, T, hidden, head.eps, x)
        ctx.fr_linear(x, headw.w, T, vocab, hidden, None, logits)
        exact = logits.double().cpu().numpy()
        for scale in (1.0, 0.7):
            a = head.logprobs(h, i32(tokens), 1, scale)
            lp.check(dict(logprobs=a["logprobs"], entropy=a["entropy"], lse=a["lse"], ids=a["top_ids"], best=a["top_logprobs"]), exact, scale, tokens, 1)
            if scale == 1.0:
                assert torch.equal(got["choice"], a["top_ids"].view(T)) and torch.equal(got["logprob"], a["top_logprobs"].view(T)) and torch.equal(got["entropy"], a["entropy"])
                assert float(a["entropy"].max() - a["entropy"].min()) > 0.01      # (not one number for all rows)
    ctx.close()
