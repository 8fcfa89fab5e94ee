"""Arrays of the paged step's calls that may not share memory: what is written beside what is read."""
import pytest
import torch

from paper_2601_12904_amd import binding as B
from tests.test_paged_host import APPEND, ARG, ATTN, TABLES, ctx, refused  # noqa: F401  (ctx is a fixture)

M = 1 << 24
FAR_APART = dict(APPEND, q=M, q_out=2 * M, k_new=3 * M, v_new=4 * M, positions=5 * M, slots=6 * M, k_pages=7 * M, v_pages=8 * M)


@pytest.mark.parametrize("name,what", [("k_new", 0), ("v_new", 16), ("k_pages", 64), ("v_pages", -16), ("positions", 0), ("slots", 20)])
def test_append_where_rotated_queries_may_not_lie(ctx, name, what):  # noqa: F811
    refused(ARG, ctx.fr_paged_append, FAR_APART, q=FAR_APART[name] // 16 * 16 + what // 16 * 16, q_out=FAR_APART[name] // 16 * 16 + what // 16 * 16)


def test_append_of_sizes_beyond_32_bits(ctx):  # noqa: F811
    refused(ARG, ctx.fr_paged_append, FAR_APART, n_tokens=2 ** 28, q=1 << 41, q_out=1 << 41, v_new=(1 << 41) + (1 << 37))


def test_append_of_arrays_side_by_side_is_not_refused(ctx):  # noqa: F811
    d, es = 64, 2 if ctx.desc.dtype == B.FR_BF16 else 4
    at, good = 1 << 20, dict(APPEND)
    for name, n in (("q", 7 * 8 * d * es), ("q_out", 7 * 8 * d * es), ("k_new", 7 * 2 * d * es), ("v_new", 7 * 2 * d * es), ("positions", 32), ("slots", 32),
                    ("k_pages", 144 * 2 * d * es), ("v_pages", 144 * 2 * d * es)):
        good[name], at = at, at + n
    if not torch.cuda.is_available():
        refused(B.FR_ERR_DEVICE, ctx.fr_paged_append, good)
        refused(B.FR_ERR_DEVICE, ctx.fr_paged_append, dict(good, q_out=good["q"]))     # in place


@pytest.mark.gpu
@pytest.mark.parametrize("name", ["q", "k_new", "v_new", "positions", "slots"])
@pytest.mark.parametrize("pages", ["k_pages", "v_pages"])
def test_append_from_within_the_pages(ctx, name, pages):  # noqa: F811
    """(Refused on the host: no kernel sees these addresses.)"""
    refused(ARG, ctx.fr_paged_append, FAR_APART, **{name: FAR_APART[pages] + 4096})


TABLES_APART = dict(TABLES, **{name: (i + 1) * M for i, name in enumerate(("cached_len", "new_len", "free_pages", "free_start", "block_table", "q_offsets", "positions", "slots", "pages_needed"))})


@pytest.mark.gpu
@pytest.mark.parametrize("written,other,at", [("pages_needed", "free_start", 0), ("pages_needed", "new_len", 8), ("q_offsets", "cached_len", -4), ("positions", "slots", 156),
                                              ("slots", "new_len", -156), ("block_table", "free_pages", 16), ("q_offsets", "block_table", 92), ("pages_needed", "positions", 156)])
def test_tables_on_top_of_one_another(ctx, written, other, at):  # noqa: F811
    """(Refused on the host: no kernel sees these addresses.)"""
    refused(ARG, ctx.fr_page_tables, TABLES_APART, **{written: TABLES_APART[other] + at})


ATTN_APART = dict(ATTN, **{name: (i + 1) * M for i, name in enumerate(("q", "q_offsets", "cached_len", "k_pages", "v_pages", "block_table", "out", "lse_out"))})


@pytest.mark.gpu
@pytest.mark.parametrize("written,other,at", [("out", "k_pages", 1024), ("out", "v_pages", -64), ("out", "block_table", 32), ("out", "q_offsets", 0), ("lse_out", "out", 64), ("lse_out", "q", 4),
                                              ("lse_out", "cached_len", 8), ("lse_out", "v_pages", 2048), ("lse_out", "q_offsets", 12)])
def test_attention_on_top_of_what_it_reads(ctx, written, other, at):  # noqa: F811
    """(Refused on the host: no kernel sees these addresses.)"""
    refused(ARG, ctx.fr_paged_attn, ATTN_APART, **{written: ATTN_APART[other] + at})
