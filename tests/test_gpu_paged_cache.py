"""GPU: PagedCache leaves its tables alone where it cannot do the whole of a
call."""
import numpy as np
import pytest

from tests.gpu_common import torch_cuda
from tests.paged_common import host, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,head_dim", [("bfloat16", 4), ("bfloat16", 36), ("float32", 6)])
def test_pages_that_cannot_be_copied_are_not_given_out(dtype, head_dim):
    """A head's row that is no multiple of 16 bytes: reserve and compact are
    refused before they change a table, a count or a length."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    from paper_2606_29223_amd.dexlib import DEX_E_INVAL, DexError
    c = paged.PagedCache(2, 1, head_dim, 4, 6, 2, 3, dtype=getattr(torch, dtype))
    c.table.copy_(ints([[3, 5, -1], [3, -1, -1]]))
    c.ref.copy_(ints([0, 0, 0, 2, 0, 1]))
    c.lens.copy_(ints([6, 3]))
    before = [host(t).copy() for t in (c.table, c.ref, c.lens)]
    for call in (lambda: c.reserve(ints([1, 1])), c.compact, lambda: c.reserve(ints([0, 0]))):
        with pytest.raises(DexError) as e:
            call()
        assert e.value.status == DEX_E_INVAL and "16 bytes" in str(e.value)
        assert all(np.array_equal(a, host(t)) for a, t in zip(before, (c.table, c.ref, c.lens)))


def test_pools_that_require_grad_are_refused_before_a_table_changes():
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    from paper_2606_29223_amd.dexlib import DexError
    c = paged.PagedCache(1, 2, 32, 4, 6, 2, 3)
    one = ints([1, 1])
    c.reserve(one)
    c.k.requires_grad_()
    before = [host(t).copy() for t in (c.table, c.ref, c.lens)]
    for call in (lambda: c.reserve(one), c.compact):
        with pytest.raises(DexError):
            call()
        assert all(np.array_equal(a, host(t)) for a, t in zip(before, (c.table, c.ref, c.lens)))
    with torch.no_grad():
        assert host(c.reserve(one).pos).tolist() == [1, 1]


def test_no_entries_are_no_copy():
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    c = paged.PagedCache(2, 2, 32, 4, 6, 2, 3)
    c.k.normal_()
    was, none = c.k.clone(), torch.empty(0, dtype=torch.int32, device="cuda")
    paged.copy(c.k, c.v, none, none)
    assert torch.equal(c.k, was)
    odd = torch.zeros((1, 2, 1, 4, 3), device="cuda")      # rows that a copy would refuse
    assert paged.copy(odd, odd, none, none) is None
