"""The entry points of trees, page selection and eviction refuse, on the host, what
their kernels would get wrong or could not be launched for; the reason is in
dex_last_error(NULL).  (The valid base arguments are never passed unchanged:
their addresses are no memory.)"""
import os

import pytest

from paper_2606_29223_amd import dexlib
from tests.test_trees_refusals import BOUNDS, EVICT, KEEP, SELECT, SPARSE, TREE, WEIGH  # noqa: F401


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(dexlib.LIB_PATH):
        pytest.skip("libdex.so not built")
    return dexlib.load()


def refused(lib, name, base, why, **change):
    assert getattr(lib, name)(*dict(base, **change).values(), None) == dexlib.DEX_E_INVAL, (name, change)
    msg = lib.dex_last_error(None).decode()
    assert msg.startswith(name + ": ") and why in msg, (msg, change)


@pytest.mark.parametrize("weight_ld,out_ld", [(6000, 6001), (6001, 6000), (5000, 1 << 40)])
def test_totals_in_place_with_another_stride_are_refused(lib, weight_ld, out_ld):
    """Workgroups would write rows that others still read."""
    refused(lib, "dex_pages_weigh", WEIGH, "another stride", weight_ld=weight_ld, weight_out_ld=out_ld)
