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


# (name, base, sizes a launch of which has 2^32 threads or a little more)
M, ROW = 1 << 20, dict(q_row=2048, o_row=2048)
TOO_MANY = [
    ("dex_pages_evict", EVICT, dict(n_seqs=M, n_kv=4, capacity=1025, weight_ld=1025, weight_out_ld=1025)),      # 1024 threads a row
    ("dex_pages_evict", EVICT, dict(n_seqs=M, n_kv=16)),                                                        # 256
    ("dex_pages_evict", EVICT, dict(n_seqs=M, n_kv=1024)),
    ("dex_pages_select", SELECT, dict(n=M, n_kv=16, n_heads=16, max_len=500)),
    ("dex_pages_select", SELECT, dict(n=1 << 14, n_kv=4, n_heads=4, max_len=1 << 15, page_size=1)),             # the scores
    ("dex_pages_bounds", BOUNDS, dict(n_seqs=1 << 22, n_kv=16, n_new=1)),
    ("dex_pages_bounds", BOUNDS, dict(n_seqs=1 << 14, max_pages=1 << 12, n_new=1 << 16, n_kv=1)),
    ("dex_pages_keep", KEEP, dict(n_seqs=1 << 20, n_layers=64, n_kv=1, capacity=5)),                            # 512 a list
    ("dex_pages_keep", KEEP, dict(n_seqs=1 << 20, n_layers=4, n_kv=1, capacity=257, index_seq=257)),            # 1024 a list
    ("dex_pages_tree_attention", TREE, dict(n=M, draft=1, n_kv=16, n_heads=16, **ROW)),
    ("dex_pages_tree_attention", TREE, dict(n=M, draft=60, n_kv=16, n_heads=16, **ROW)),
    ("dex_pages_sparse_attention", SPARSE, dict(n=M, n_kv=16, n_heads=16, q_row=1024, o_row=1024, head_dim=32, o_head=32, n_columns=9)),
    ("dex_pages_sparse_attention", SPARSE, dict(n=M, n_kv=32, n_heads=32, **ROW)),
    ("dex_pages_weigh", WEIGH, dict(n=M, n_kv=16, n_heads=16, max_len=300, q_row=1024, o_row=1024, head_dim=32, o_head=32)),
    ("dex_pages_weigh", WEIGH, dict(n=1 << 17, n_kv=16, n_heads=16, max_len=8192, weight_ld=8192, weight_out_ld=8192, **ROW)),   # the weights
]


@pytest.mark.parametrize("i", range(len(TOO_MANY)))
def test_launches_of_too_many_threads_are_refused(lib, i):
    name, base, change = TOO_MANY[i]
    refused(lib, name, base, "2^32 threads", **change)


def test_work_of_sizes_that_are_refused_is_none(lib):
    """The bytes of these do not fit in 64 bits."""
    assert lib.dex_pages_weigh_work(1, M, 8192, 128, 128, 1 << 30) == 0
    assert lib.dex_pages_weigh_work(1, M, 8192, 128, 128, 100) == 0
    assert lib.dex_pages_select_work(M, 4096, 1, (1 << 31) - 1) == 0
    assert lib.dex_pages_weigh_work(1, 4, 32, 8, 128, 1 << 20) > 4 * 32 * (1 << 20) * 4
    assert lib.dex_pages_select_work(64, 8, 16, 1 << 20) == 64 * 8 * (1 << 16) * 8
