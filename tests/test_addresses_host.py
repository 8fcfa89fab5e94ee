"""Raw addresses in the place of tensors: whole numbers of any kind that Python knows as int."""
import enum

import pytest
import torch

from paper_2601_12904_amd import binding as B


class Address(int):
    pass


class Buffer(enum.IntEnum):
    PAGES = 1 << 20


@pytest.mark.parametrize("at", [1 << 20, Address(1 << 20), Buffer.PAGES])
def test_whole_numbers_are_addresses(at):
    assert B._ptr(at) == 1 << 20
    assert B._rows(at, 5, 8, 64) == (1 << 20, 512)
    assert B.pointers([at, None, at]).tolist() == [1 << 20, 0, 1 << 20]


@pytest.mark.parametrize("at", [Address(1 << 40), Buffer.PAGES])
def test_calls_take_them(at):
    """(They get as far as the library's own checks: an address that is not aligned.)"""
    ctx = B.Context(8, 2, 64, B.FR_BF16, 1e4, max_tokens=64, max_chunks=1, max_question_tokens=1)
    for call in (lambda: ctx.fr_rmsnorm(Address(at + 8), at, 4, 256, 1e-5, at), lambda: ctx.fr_qk_norm_append(None, Address(at + 8), at, at, at, 1e-5, None, None, 1, at, at, 1, 1)):
        with pytest.raises(B.FusionRAGError) as e:
            call()
        assert e.value.status == B.FR_ERR_INVALID_ARG
    ctx.close()


def test_tensors_with_gaps_are_not():
    with pytest.raises(ValueError):
        B._ptr(torch.zeros(4, 4)[:, :2])
