"""Host-side checks of the paged step's entry points: refusals before anything reaches a device."""
import pytest
import torch

from paper_2601_12904_amd import binding as B

P = 4096   # an aligned, non-null device address: validation must fail before any launch


@pytest.fixture(params=[B.FR_BF16, B.FR_F32])
def ctx(request):
    c = B.Context(8, 2, 64, request.param, 1e4, max_tokens=64, max_chunks=1, max_question_tokens=1)
    yield c
    c.close()


def refused(status, fn, good, **change):
    with pytest.raises(B.FusionRAGError) as e:
        fn(**{**good, **change})
    assert e.value.status == status, str(e.value)
    assert len(str(e.value)) > 25                        # says what is wrong


TABLES = dict(cached_len=P, new_len=P, n_requests=3, page_rows=16, free_pages=P, n_free=5, free_start=P, block_table=P, max_blocks=8,
              n_tokens=40, q_offsets=P, positions=P, slots=P, pages_needed=P)
APPEND = dict(q=P, k_new=P, v_new=P, positions=P, slots=P, n_tokens=7, k_pages=P, v_pages=P, n_pages=9, page_rows=16, q_out=P + 2 ** 20)
ATTN = dict(q=P, q_offsets=P, cached_len=P, n_requests=3, n_tokens=7, max_new=5, k_pages=P, v_pages=P, n_pages=9, page_rows=16,
            block_table=P, max_blocks=8, out=P, lse_out=P)
ARG, UNS = B.FR_ERR_INVALID_ARG, B.FR_ERR_UNSUPPORTED


@pytest.mark.parametrize("status,change", [
    (ARG, dict(n_requests=-1)), (UNS, dict(n_requests=B.FR_PAGED_MAX_REQUESTS + 1)), (ARG, dict(page_rows=0)), (ARG, dict(max_blocks=-1)),
    (UNS, dict(max_blocks=2 ** 27)), (ARG, dict(n_tokens=-1)), (UNS, dict(n_tokens=2 ** 30 + 1)), (ARG, dict(n_free=-1)), (ARG, dict(cached_len=None)),
    (ARG, dict(new_len=P + 2)), (ARG, dict(free_pages=None)), (ARG, dict(block_table=None)), (ARG, dict(q_offsets=None)), (ARG, dict(positions=None)),
    (ARG, dict(slots=P + 1)), (ARG, dict(free_start=P + 3)), (ARG, dict(pages_needed=P + 2))])
def test_tables_refusals(ctx, status, change):
    refused(status, ctx.fr_page_tables, TABLES, **change)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(n_tokens=-1)), (UNS, dict(n_tokens=2 ** 30 + 1)), (ARG, dict(n_pages=-1)), (ARG, dict(page_rows=0)), (UNS, dict(n_pages=2 ** 27)),
    (ARG, dict(k_new=None)), (ARG, dict(v_new=P + 8)), (ARG, dict(k_pages=None)), (ARG, dict(v_pages=P + 4)), (ARG, dict(slots=None)),
    (ARG, dict(positions=P + 2)), (ARG, dict(q_out=None)), (ARG, dict(q=None)), (ARG, dict(q=P + 8, q_out=P + 8)), (ARG, dict(positions=None)),
    (ARG, dict(q_out=P + 64))])
def test_append_refusals(ctx, status, change):
    refused(status, ctx.fr_paged_append, APPEND, **change)


@pytest.mark.parametrize("status,change", [
    (ARG, dict(n_requests=-1)), (UNS, dict(n_requests=B.FR_PAGED_MAX_REQUESTS + 1)), (ARG, dict(page_rows=-1)), (ARG, dict(max_blocks=-1)),
    (UNS, dict(max_blocks=2 ** 26 + 1)), (ARG, dict(n_tokens=-1)), (ARG, dict(n_pages=-1)), (UNS, dict(n_pages=2 ** 27)), (ARG, dict(max_new=-1)),
    (ARG, dict(q=None)), (ARG, dict(out=P + 8)), (ARG, dict(k_pages=P + 2)), (ARG, dict(v_pages=None)), (ARG, dict(q_offsets=None)),
    (ARG, dict(cached_len=P + 1)), (ARG, dict(block_table=None)), (ARG, dict(lse_out=P + 2))])
def test_attention_refusals(ctx, status, change):
    refused(status, ctx.fr_paged_attn, ATTN, **change)


def test_rows_times_heads_stay_below_two_to_the_31(ctx):
    refused(UNS, ctx.fr_paged_attn, ATTN, n_tokens=2 ** 28)         # eight heads


def test_outputs_on_top_of_queries_only_as_a_whole(ctx):
    refused(ARG, ctx.fr_paged_attn, ATTN, out=P + 256)
    refused(ARG, ctx.fr_paged_attn, ATTN, q=P + 256)


def test_option_values(ctx):
    for v in (B.FR_PAGED_KERNEL_AUTO, B.FR_PAGED_KERNEL_STREAM, B.FR_PAGED_KERNEL_TILED):
        ctx.fr_set_option(B.FR_OPT_PAGED_KERNEL, v)
    refused(ARG, ctx.fr_set_option, dict(option=B.FR_OPT_PAGED_KERNEL), value=3)


def test_nothing_to_do(ctx):
    ctx.fr_paged_append(**{**APPEND, "n_tokens": 0, "k_new": None, "slots": None})
    for none in ("n_tokens", "n_requests", "max_new"):
        ctx.fr_paged_attn(**{**ATTN, none: 0, "q": None, "out": None})


def test_tensors_have_to_be_contiguous(ctx):
    with pytest.raises(ValueError):
        ctx.fr_paged_attn(**{**ATTN, "q": torch.zeros(7, 8, 128)[:, :, :64]})


def test_a_valid_call_without_a_gpu_is_a_device_error(ctx):
    if torch.cuda.is_available():
        pytest.skip("a GPU is present")
    for fn, good in ((ctx.fr_page_tables, TABLES), (ctx.fr_paged_append, APPEND), (ctx.fr_paged_attn, ATTN)):
        refused(B.FR_ERR_DEVICE, fn, good)
