"""The entry points of trees, page selection and eviction refuse bad arguments
on the host, before any device call, with the reason in dex_last_error(NULL);
the binding refuses tensors that do not fit, and those whose gradients it would
lose.  (The valid base arguments are never passed unchanged: their addresses are
no memory.)"""
import math
import os

import pytest

from paper_2606_29223_amd import dexlib, paged

torch = pytest.importorskip("torch")
from torch.autograd import forward_ad  # noqa: E402

FAKE = 0x1000


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(dexlib.LIB_PATH):
        pytest.skip("libdex.so not built")
    return dexlib.load()


MASK = dict(parent=FAKE, n_trees=2, draft=9, mask=FAKE, depth=FAKE)
ACCEPT = dict(parent=FAKE, token=FAKE, target=FAKE, n_draft=None, root=None, n_trees=2, draft=9, path=FAKE, count=FAKE,
              next=FAKE)
PAGES = dict(k_pages=FAKE, v_pages=FAKE, n_pages=80, page_size=16, table=FAKE, n_seqs=2, max_pages=400)
OUT = dict(out=FAKE, o_row=256, o_head=64, lse=None, work=FAKE)
QUERY = dict(q=FAKE, q_row=256, q_head=64)
TREE = dict(dtype=1, head_dim=64, n_heads=4, n_kv=2, n=2, draft=9, seq=None, lens=FAKE, drafts=None, max_len=5000, scale=0.125,
            **QUERY, mask=FAKE, **PAGES, **OUT)
SPARSE = dict(dtype=1, head_dim=64, n_heads=4, n_kv=2, n=2, seq=None, lens=FAKE, scale=0.125, **QUERY, columns=FAKE,
              n_columns=99, **PAGES, **OUT)
WEIGH = dict(dtype=1, head_dim=64, n_heads=4, n_kv=2, n=2, seq=None, lens=FAKE, max_len=5000, scale=0.125, **QUERY, weight=FAKE,
             weight_ld=6000, weight_out=FAKE, weight_out_ld=6000, **PAGES, **OUT)
KEEP = dict(dtype=1, head_dim=64, n_layers=2, n_pages=8, n_kv=2, page_size=16, k=FAKE, v=FAKE, table=FAKE, n_seqs=2, max_pages=4,
            to=None, to_pages=0, first=None, index=FAKE, index_layer=0, index_seq=5, index_head=0, capacity=5, count=FAKE)
TRIM = dict(table=FAKE, ref=FAKE, length=FAKE, n_seqs=2, max_pages=4, n_pages=8, page_size=16, t=FAKE, r=FAKE)
BOUNDS = dict(dtype=1, head_dim=64, k_pages=FAKE, n_pages=8, n_kv=2, page_size=16, table=FAKE, n_seqs=2, max_pages=4, length=FAKE,
              n_new=3, bounds=FAKE)
SELECT = dict(dtype=1, head_dim=64, n_heads=4, n_kv=2, n=2, seq=None, lens=FAKE, max_len=5000, **QUERY, bounds=FAKE, n_pages=80,
              page_size=16, table=FAKE, n_seqs=2, max_pages=400, n_select=8, sinks=1, recent=2, columns=FAKE, work=FAKE)
EVICT = dict(weight=FAKE, weight_ld=900, n_seqs=2, n_kv=3, capacity=900, length=FAKE, budget=100, sinks=4, recent=10, index=FAKE,
             count=FAKE, weight_out=FAKE, weight_out_ld=900)

CACHE = [(dict(dtype=2), "dtype"), (dict(head_dim=63), "head_dim"), (dict(page_size=24), "power of two"),
         (dict(page_size=0), "power of two"), (dict(n_pages=0), "n_pages"), (dict(n_pages=1 << 30), "2^32"),
         (dict(n_kv=0), "n_kv_heads"), (dict(n_seqs=0), "n_seqs"), (dict(max_pages=0), "max_pages"),
         (dict(max_pages=1 << 28), "position")]
HEADS = [(dict(head_dim=96), "head_dim"), (dict(n_heads=3), "multiple"), (dict(n_heads=1), "multiple"),
         (dict(n_heads=130), "64 times"), (dict(n_heads=8320, n_kv=260), "8192"), (dict(n=-1), "2^20"), (dict(n=(1 << 20) + 1), "2^20"),
         (dict(n=1 << 20, n_heads=8192, n_kv=512), "too many")]
ATTENTION = HEADS + [(dict(scale=math.inf), "scale"), (dict(scale=math.nan), "scale"), (dict(q=None), "NULL"),
                     (dict(lens=None), "NULL"), (dict(out=None), "NULL"), (dict(table=None), "NULL"), (dict(v_pages=None), "NULL"),
                     (dict(work=None), "work"), (dict(work=FAKE + 4), "work"), (dict(k_pages=FAKE + 8), "aligned"),
                     (dict(lse=FAKE + 2), "aligned to"), (dict(seq=FAKE + 2), "aligned to"), (dict(q=FAKE + 1), "aligned to"),
                     (dict(out=FAKE + 1), "aligned to"), (dict(lens=FAKE + 1), "aligned to"), (dict(table=FAKE + 2), "aligned to")]
ATTENTION += [(dict(zip(("o_row", "o_head"), st)), "overlap") for st in
              [(0, 64), (1 << 20, 0), (63, 128), (1 << 20, 63), (-1, 64), (64, 64), (-2 ** 63, 1)]]
BIG = 1 << 30
BAD = (
    [("dex_tree_mask", MASK, *b) for b in [
        (dict(n_trees=-1), "n_trees"), (dict(n_trees=(1 << 20) + 1), "n_trees"), (dict(draft=0), "draft"), (dict(draft=257), "draft"),
        (dict(parent=None), "NULL"), (dict(mask=None), "NULL"), (dict(mask=FAKE + 4), "aligned"), (dict(parent=FAKE + 2), "aligned"),
        (dict(depth=FAKE + 1), "aligned")]]
    + [("dex_tree_accept", ACCEPT, *b) for b in [
        (dict(n_trees=-1), "n_trees"), (dict(draft=0), "draft"), (dict(draft=257), "draft")]
        + [({n: None}, "NULL") for n in ("parent", "token", "target", "path", "count", "next")]
        + [({n: FAKE + 2}, "aligned") for n in ("parent", "token", "target", "path", "count", "next", "n_draft", "root")]]
    + [("dex_pages_tree_attention", TREE, *b) for b in CACHE + ATTENTION + [
        (dict(draft=0), "draft"), (dict(draft=257), "draft"), (dict(max_len=-1), "max_len"), (dict(max_len=BIG + 1), "max_len"),
        (dict(mask=None), "mask"), (dict(mask=FAKE + 4), "aligned"), (dict(drafts=FAKE + 2), "aligned"),
        (dict(n=1 << 20, draft=256, n_heads=6), "too many")]]
    + [("dex_pages_sparse_attention", SPARSE, *b) for b in CACHE + ATTENTION + [
        (dict(n_columns=0), "n_columns"), (dict(n_columns=(1 << 26) + 1), "n_columns"), (dict(columns=None), "NULL"),
        (dict(columns=FAKE + 2), "aligned")]]
    + [("dex_pages_weigh", WEIGH, *b) for b in CACHE + ATTENTION + [
        (dict(max_len=-1), "max_len"), (dict(max_len=6001), "shorter"), (dict(weight_ld=4999), "shorter"),
        (dict(weight_out_ld=4999), "shorter"), (dict(weight=None), "NULL"), (dict(weight_out=None), "NULL"),
        (dict(weight=FAKE + 2), "aligned"), (dict(weight_out=FAKE + 2), "aligned"),
        (dict(n=1 << 14, max_len=BIG, weight_ld=BIG, weight_out_ld=BIG), "too many")]]
    + [("dex_pages_keep", KEEP, *b) for b in CACHE[:7] + [(dict(n_seqs=0), "n_seqs"), (dict(max_pages=0), "max_pages")] + [
        (dict(head_dim=4), "16 bytes"), (dict(n_layers=0), "n_layers"), (dict(n_layers=(1 << 19) + 1), "n_layers"),
        (dict(n_seqs=1 << 20, n_layers=1 << 10), "too many"), (dict(to=FAKE), "to_pages"), (dict(to=FAKE, to_pages=1 << 27), "to_pages"),
        (dict(capacity=-1), "capacity"), (dict(capacity=BIG + 1), "capacity"), (dict(index_layer=-1), "stride"),
        (dict(index_seq=-1), "stride"), (dict(index_head=-1), "stride"), (dict(k=None), "NULL"), (dict(v=None), "NULL"),
        (dict(table=None), "NULL"), (dict(index=None), "NULL"), (dict(count=None), "NULL"), (dict(k=FAKE + 8), "aligned"),
        (dict(v=FAKE + 2), "aligned"), (dict(table=FAKE + 2), "aligned"), (dict(index=FAKE + 1), "aligned"),
        (dict(count=FAKE + 2), "aligned"), (dict(first=FAKE + 2), "aligned"), (dict(to=FAKE + 2, to_pages=4), "aligned")]]
    + [("dex_pages_trim", TRIM, *b) for b in [(dict(n_seqs=0), "n_seqs"), (dict(max_pages=0), "max_pages"),
                                              (dict(max_pages=1 << 28), "position"), (dict(n_pages=0), "n_pages"),
                                              (dict(n_pages=BIG + 1), "n_pages"), (dict(page_size=3), "power of two")]
       + [({n: None}, "NULL") for n in ("table", "ref", "length", "t", "r")]
       + [({n: FAKE + 2}, "aligned") for n in ("table", "ref", "length", "t", "r")]]
    + [("dex_pages_bounds", BOUNDS, *b) for b in CACHE + [
        (dict(head_dim=96), "head_dim"), (dict(n_new=-1), "n_new"), (dict(k_pages=None), "NULL"), (dict(table=None), "NULL"),
        (dict(length=None), "NULL"), (dict(bounds=None), "NULL"), (dict(k_pages=FAKE + 8), "aligned"), (dict(bounds=FAKE + 8), "aligned"),
        (dict(table=FAKE + 2), "aligned"), (dict(length=FAKE + 2), "aligned"),
        (dict(n_seqs=1 << 24, max_pages=1 << 20, n_new=1 << 20), "too many")]]
    + [("dex_pages_select", SELECT, *b) for b in CACHE + HEADS + [
        (dict(max_len=-1), "max_len"), (dict(sinks=-1), "sinks"), (dict(recent=-1), "sinks"), (dict(n_select=2), "n_select"),
        (dict(n_select=0, sinks=0, recent=0), "n_select"), (dict(q=None), "NULL"), (dict(bounds=None), "NULL"), (dict(table=None), "NULL"),
        (dict(lens=None), "NULL"), (dict(columns=None), "NULL"), (dict(work=None), "work"), (dict(work=FAKE + 8), "work"),
        (dict(bounds=FAKE + 8), "aligned"), (dict(q=FAKE + 1), "aligned"), (dict(seq=FAKE + 2), "aligned"), (dict(lens=FAKE + 2), "aligned"),
        (dict(columns=FAKE + 2), "aligned"), (dict(n=1 << 20, max_len=BIG), "too many")]]
    + [("dex_pages_evict", EVICT, *b) for b in [
        (dict(n_seqs=-1), "n_seqs"), (dict(n_kv=0), "n_kv_heads"), (dict(n_kv=4097), "n_kv_heads"), (dict(capacity=0), "capacity"),
        (dict(n_seqs=1 << 20, n_kv=4096), "too many"), (dict(sinks=-1), "sinks"), (dict(recent=-1), "sinks"), (dict(budget=13), "budget"),
        (dict(budget=0, sinks=0, recent=0), "budget"), (dict(weight_ld=899), "shorter"), (dict(weight_out_ld=899), "shorter"),
        (dict(weight_out_ld=901), "stride")]
        + [({n: None}, "NULL") for n in ("weight", "length", "index", "count", "weight_out")]
        + [({n: FAKE + 2}, "aligned") for n in ("weight", "length", "index", "count", "weight_out")]]
)


@pytest.mark.parametrize("i", range(len(BAD)))
def test_bad_arguments_are_refused(lib, i):
    name, base, change, why = BAD[i]
    assert getattr(lib, name)(*dict(base, **change).values(), None) == dexlib.DEX_E_INVAL, (name, change)
    msg = lib.dex_last_error(None).decode()
    assert msg.startswith(name + ": ") and why in msg, (msg, change)


def test_nothing_to_do_is_no_work(lib):
    for name, base, change in (("dex_tree_mask", MASK, dict(n_trees=0)), ("dex_tree_accept", ACCEPT, dict(n_trees=0)),
                               ("dex_pages_tree_attention", TREE, dict(n=0)), ("dex_pages_sparse_attention", SPARSE, dict(n=0)),
                               ("dex_pages_weigh", WEIGH, dict(n=0)), ("dex_pages_keep", KEEP, dict(capacity=0)),
                               ("dex_pages_bounds", BOUNDS, dict(n_new=0)), ("dex_pages_select", SELECT, dict(n=0)),
                               ("dex_pages_evict", EVICT, dict(n_seqs=0))):
        assert getattr(lib, name)(*dict(base, **change).values(), None) == dexlib.DEX_OK, name


def test_work_sizes(lib):
    small, big = (lib.dex_pages_tree_attention_work(1, 4, 8, 32, 8, 128, n) for n in (100, 65536))
    assert 0 <= small < big
    assert lib.dex_pages_tree_attention_work(1, 4, 8, 32, 8, 128, 1 << 30) < 1 << 32
    assert lib.dex_pages_tree_attention_work(1, 64, 64, 32, 8, 128, 1 << 20) < 1 << 32
    assert lib.dex_pages_weigh_work(1, 4, 32, 8, 128, 5000) >= 4 * 32 * 5000 * 4
    assert lib.dex_pages_select_work(4, 8, 16, 1601) == 4 * 8 * 101 * 8
    for bad in ((7, 4, 8, 32, 8, 128, 100), (1, 4, 257, 32, 8, 128, 100), (1, -4, 8, 32, 8, 128, 100), (1, 4, 8, 32, 8, 96, 100),
                (1, 4, 8, 32, 0, 128, 100), (1, 4, 8, 32, 8, 128, -1)):
        assert lib.dex_pages_tree_attention_work(*bad) == 0
    assert lib.dex_pages_sparse_attention_work(1, 4, 32, 8, 128, 64, 17) == 0
    assert lib.dex_pages_weigh_work(1, 4, 32, 8, 128, -1) == 0 and lib.dex_pages_select_work(4, 8, 3, 100) == 0


def _tensors():
    t = {n: torch.zeros((2, 2, 32)) for n in ("q", "out")}
    t.update({n: torch.zeros((4, 2, 4, 32)) for n in ("k_pages", "v_pages")})
    t.update(bounds=torch.zeros((4, 2, 2, 32)), weight=torch.zeros((2, 2, 8)), weight_out=torch.zeros((2, 2, 8)))
    return t


N, TABLE = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)
COLUMNS, BITS = torch.zeros((2, 2, 2), dtype=torch.int32), torch.zeros((2, 1, 1), dtype=torch.int64)
CALLS = {
    "tree_attention": (lambda q, k_pages, v_pages, out, **_: paged.tree_attention(q, k_pages, v_pages, TABLE, N, BITS, out=out),
                       "q k_pages v_pages out"),
    "keep": (lambda k_pages, v_pages, **_: paged.keep(k_pages[None], v_pages[None], TABLE, TABLE, N), "k_pages v_pages"),
    "page_bounds": (lambda k_pages, bounds, **_: paged.page_bounds(k_pages, TABLE, N, out=bounds), "k_pages bounds"),
    "select_pages": (lambda q, bounds, **_: paged.select_pages(q, bounds, TABLE, N, 4, 2), "q bounds"),
    "sparse_attention": (lambda q, k_pages, v_pages, out, **_: paged.sparse_attention(q, k_pages, v_pages, TABLE, N, COLUMNS, out=out),
                         "q k_pages v_pages out"),
    "weigh": (lambda q, k_pages, v_pages, weight, weight_out, out, **_: paged.weigh(
        q, k_pages, v_pages, TABLE, N, weight, weight_out=weight_out, out=out), "q k_pages v_pages weight weight_out out"),
    "evict": (lambda weight, weight_out, **_: paged.evict(weight, N, 3, weight_out=weight_out), "weight weight_out"),
}
WHICH = [(call, name) for call, (_, names) in CALLS.items() for name in names.split()]


@pytest.mark.parametrize("call,name", WHICH)
def test_a_tensor_that_requires_grad_is_refused(call, name):
    x = _tensors()
    x[name].requires_grad_()
    with pytest.raises(dexlib.DexError, match="requires grad"):
        CALLS[call][0](**x)
    with torch.no_grad(), pytest.raises(dexlib.DexError, match="GPU"):
        CALLS[call][0](**x)


@pytest.mark.parametrize("call,name", WHICH)
def test_a_tensor_with_a_tangent_is_refused(call, name):
    x = _tensors()
    with forward_ad.dual_level():
        x[name] = forward_ad.make_dual(x[name], torch.ones_like(x[name]))
        with pytest.raises(dexlib.DexError, match="tangent"):
            CALLS[call][0](**x)


def test_the_binding_refuses_tensors_off_the_gpu():
    parent = torch.zeros((2, 3), dtype=torch.int32)
    for call in (lambda: paged.tree_mask(parent), lambda: paged.tree_accept(parent, parent, parent), lambda: paged.trim(TABLE, N, N, 4)):
        with pytest.raises(dexlib.DexError) as e:
            call()
        assert e.value.status == dexlib.DEX_E_INVAL


def test_a_cache_without_bounds_says_so():
    cache = paged.PagedCache(1, 2, 32, 4, 4, 2, 2, device="cpu")
    for call in (lambda: cache.update_bounds(0), lambda: cache.sparse_attention(0, torch.zeros((2, 2, 32)), 2)):
        with pytest.raises(dexlib.DexError, match="bounds"):
            call()
    with pytest.raises(dexlib.DexError, match="weight"):
        cache.evict(torch.zeros((2, 2, 8)), 4)
