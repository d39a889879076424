"""Rotary positions at the C boundary, without a GPU: what else is refused before any HIP call."""
import pytest
import torch

from paper_2605_05699_amd import binding as B
from tests.test_paged_abi import rotary


@pytest.fixture(scope="module")
def L():
    return B.lib()


def test_rotary_in_place_takes_one_type_and_one_layout(L):
    here = 1 << 20
    for other in (dict(out_type=2), dict(in_type=0, out_type=1), dict(out_token=256), dict(out_head=72), dict(in_token=0), dict(in_head=0)):
        assert rotary(L, out_dev=here, **other) == -7, other


def test_rotary_rows_of_a_token_are_counted_with_32_bits(L):
    for over in (dict(n_heads=1 << 25), dict(n_heads=1 << 21, d=1024, rot=1024), dict(n_heads=(1 << 30) - 1, d=2, rot=2, tokens=3)):
        assert rotary(L, **dict(dict(tokens=1), **over)) == -7, over


class _Device(torch.Tensor):
    """A host tensor that says it is on the device: nothing here reads it there."""
    is_cuda = property(lambda self: True)


@pytest.mark.parametrize("bounds", [dict(max_new=1 << 32), dict(max_new=(1 << 32) + 1), dict(max_new=-1), dict(max_length=1 << 64), dict(max_length=-5)])
def test_bounds_that_the_structure_cannot_hold_are_refused(bounds):
    """(c_int32 keeps the low 32 bits of what it is given: a bound of 2^32 cut every token off.)"""
    table, windows, lengths, starts = (torch.zeros(s, dtype=torch.int32).as_subclass(_Device) for s in ((2, 3), (2, 2), (2,), (3,)))
    B.PagedSeqs(table, windows, lengths, starts, max_new=(1 << 31) - 1, max_length=16)
    with pytest.raises(ValueError):
        B.PagedSeqs(table, windows, lengths, starts, **dict(dict(max_new=1, max_length=16), **bounds))
