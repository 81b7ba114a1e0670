"""Operators over a paged key/value cache on torch tensors (include/dex.h,
same names): rotary positions and the cache write, attention of one new token
a row, page tables that fork, grow and compact, beam selection; trees of drafted
tokens, attention over chosen pages, and eviction by accumulated weight.

A cache is plain tensors of the caller: a layer's keys and values are
[n_pages, n_kv_heads, page_size, head_dim] each, a pool of layers
[n_layers, ...] of those; `table` [n_seqs, max_pages] lists each sequence's
pages (-1: none), `ref` [n_pages] counts their holders, `lens` [n_seqs] the
sequences' tokens (int32).  `PagedCache` holds them together.

Every function enqueues on the tensors' device, on the stream that is current
there, and waits for nothing: calls can be captured into a graph.  Outputs and
work memory come from torch's allocator, call by call; an output of the
caller's overlaps no input unless the function says that it may.  Bad arguments
raise `DexError` before anything is launched.  Nothing is recorded for
autograd: a tensor that requires grad while grad mode is on, or that carries a
forward-mode tangent, is refused (torch.no_grad, or detach), and an output of
the caller's keeps its version.  `rope` with `inverse` is the gradient of `rope`.

A step of a decoding loop with branches, for a model of the caller's:

    pos = cache.reserve(n_new).pos                     # room for the next tokens
    for layer in range(cache.n_layers):
        q = cache.append(layer, pos, q, k, v, rotary)  # rotate and write
        out = cache.attention(layer, q, group=beams)
    parent, token, score, done = paged.beam_select(logits, score, done=done, eos=eos)
    cache.fork(parent.flatten())                      # the branches follow their parents

A step with drafted tokens, up to `draft` of them a sequence in trees (a
sequence that reserve grants nothing, asked for or not, stays as it is):

    mask, depth = paged.tree_mask(parent)
    before = cache.lens.clone()
    place = cache.reserve(n_draft).places(draft).flatten()   # n_draft: each tree's tokens, 0 to draft
    granted = cache.lens - before                      # n_draft, or 0
    at = (before[:, None] + depth).flatten()           # rotary positions
    for layer in range(cache.n_layers):
        q, k = paged.rope(rotary, at, q, k)
        cache.append(layer, place, q, k, v, seq=seq)   # seq: each row's sequence
        out = cache.tree_attention(layer, q, before, mask, n_draft=granted)
    path, count, token = paged.tree_accept(parent, drafted, target, n_draft=granted, root=token)
    cache.accept(before, path, count)                  # the path's tokens stay, the others go

Here every tree's first node is its sequence's last token, `token`, which stays
the next one where nothing was granted.
"""

from __future__ import annotations

import ctypes
import functools
import math
from typing import NamedTuple

import torch
from torch.autograd import forward_ad

from . import dexlib
from .dexlib import DEX_BF16, DEX_E_INVAL, DEX_F32, DexError

SCALING = {None: 0, "linear": 1, "base": 2, "bands": 3}
_DTYPES = {torch.float32: DEX_F32, torch.bfloat16: DEX_BF16}
_grad_enabled = torch.is_grad_enabled


def _refuse(why: str):
    raise DexError(DEX_E_INVAL, why)


# (Written out: with `any` the two checks take 0.5 us of a small call's 13.)
def _detached(*tensors):
    """Refuses tensors whose gradients or tangents a call would lose."""
    if _grad_enabled():
        for t in tensors:
            if t is not None and t.requires_grad:
                _refuse("a tensor requires grad, and nothing is recorded for autograd")
    if getattr(forward_ad, "_current_level", 0) >= 0:     # inside a dual_level
        for t in tensors:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                _refuse("a tensor carries a tangent, and nothing is recorded for autograd")


# The current stream's handle: torch's own short cut to it where it has one
# (0.1 us a call; building a Stream object takes 2 to 3 of a small call's 12).
_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)


# Work memory by a call's sizes, asked once for each (0.6 us of a small call's 17).
@functools.lru_cache(maxsize=4096)
def _attention_work(*sizes):
    return dexlib.load().dex_pages_attention_work(*sizes)


@functools.lru_cache(maxsize=4096)
def _beam_work(*sizes):
    return max(16, dexlib.load().dex_beam_select_work(*sizes))


def _run(fn, device, *args):
    """One library call on the current stream of `device`."""
    i = device.index
    if i == torch.cuda.current_device():
        st = fn(*args, _stream(i))
    else:
        with torch.cuda.device(device):
            st = fn(*args, _stream(i))
    if st:
        m = dexlib.load().dex_last_error(None)
        raise DexError(st, m.decode() if m else "")


def _ints(t, device, shape, name):
    """A contiguous int32 tensor of the given shape on the device: its address."""
    if t.dtype is not torch.int32 or t.device != device or t.shape != shape or not t.is_contiguous():
        _refuse(f"{name}: a contiguous int32 tensor of shape {tuple(shape)} on {device} is wanted, "
                f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _heads(t, device, dtype, shape, name):
    """[rows, heads, head_dim], its last dimension dense: address and strides."""
    if t.dtype is not dtype or t.device != device or t.shape != shape:
        _refuse(f"{name}: {dtype} of shape {tuple(shape)} on {device} is wanted, "
                f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return _strided(t, name)


def _strided(t, name):
    r, h, d = t.stride()
    if d != 1 and t.shape[2] > 1:
        _refuse(f"{name}: head_dim has to be dense")
    return t.data_ptr(), r, h


def _out(t, like, shape, name):
    """The caller's output, checked, or a new one: (tensor, address and strides)."""
    if t is not None:
        return t, _heads(t, like.device, like.dtype, shape, name)
    t = like.new_empty(shape)
    return t, (t.data_ptr(), shape[1] * shape[2], shape[2])


def _gpu(t, name):
    """dex_dtype of a floating GPU tensor."""
    if t.device.type != "cuda":
        _refuse(f"{name} is not on a GPU")
    d = _DTYPES.get(t.dtype)
    if d is None:
        _refuse(f"{name}: {t.dtype} is neither float32 nor bfloat16")
    return d


def _pages(k, v, table, name="k_pages"):
    """Checks one layer's pages and their table; the layer's sizes."""
    d = _gpu(k, name)
    if k.dim() != 4 or not k.is_contiguous():
        _refuse(f"{name}: a contiguous [n_pages, n_kv_heads, page_size, head_dim] is wanted, got {tuple(k.shape)}")
    if v.dtype is not k.dtype or v.device != k.device or v.shape != k.shape or not v.is_contiguous():
        _refuse("values and keys differ in type, device or shape")
    if table.dim() != 2:
        _refuse("table is [n_seqs, max_pages]")
    return d, k.shape


class Rotary:
    """A plan of rotary positions (dex_rotary): `rot_dim` leading dimensions of
    each head turn (all by default), pairs half a turned part apart or
    neighbours (`interleaved`).  scaling: None, "linear" (frequencies divided
    by `factor`), "base" (theta raised so that the lowest is divided by it) or
    "bands" (those that make at most `slow` turns over `original` positions
    are, those that make at least `fast` are not).  `amplitude` multiplies
    cosine and sine."""

    def __init__(self, head_dim, rot_dim=None, theta=1e4, interleaved=False, scaling=None, factor=1.0, original=0.0,
                 slow=1.0, fast=32.0, amplitude=1.0, device="cuda"):
        self.head_dim = int(head_dim)
        self.rot_dim = int(head_dim if rot_dim is None else rot_dim)
        if scaling not in SCALING:
            _refuse(f"unknown scaling {scaling!r}")
        if not 2 <= self.rot_dim <= self.head_dim:
            _refuse("rot_dim is not 2 to head_dim")
        turns = (ctypes.c_double * (self.rot_dim // 2))()
        lib = dexlib.load()
        dexlib._check(lib, None, lib.dex_rotary_turns(SCALING[scaling], self.rot_dim, theta, factor, original, slow, fast,
                                                      turns))
        self.turns = torch.frombuffer(turns, dtype=torch.float64).to(device, copy=True)
        self.struct = dexlib.DexRotary(self.turns.data_ptr(), self.rot_dim, int(bool(interleaved)), float(amplitude))


def _plan(rotary, device, head_dim):
    if rotary.turns.device != device or rotary.head_dim != head_dim:
        _refuse(f"the rotary plan is for head_dim {rotary.head_dim} on {rotary.turns.device}")
    return rotary.struct


def rope(rotary, pos, q, k=None, q_out=None, k_out=None, inverse=False):
    """Queries (and keys) [rows, heads, head_dim] turned to positions `pos`
    [rows] int32; `inverse` turns back (the gradient of the turn).  An output
    may be its input.  Returns q_out, or (q_out, k_out)."""
    _detached(q, k, q_out, k_out)
    d = _gpu(q, "q")
    dev, dt = q.device, q.dtype
    if q.dim() != 3 or (k is not None and k.dim() != 3):
        _refuse("queries and keys are [rows, heads, head_dim]")
    rows, heads, hd = q.shape
    plan = _plan(rotary, dev, hd)
    a = _strided(q, "q")
    q_out, b = _out(q_out, q, (rows, heads, hd), "q_out")
    n, c, o = 0, (None, 0, 0), (None, 0, 0)
    if k is not None:
        n = k.shape[1]
        c = _heads(k, dev, dt, (rows, n, hd), "k")
        k_out, o = _out(k_out, q, (rows, n, hd), "k_out")
    p = _ints(pos, dev, (rows,), "pos")
    if rows > 0:
        _run(dexlib.load().dex_rope, dev, d, hd, plan, 1 if inverse else 0, rows, p, *a, heads, *b, *c, n, *o)
    return q_out if k is None else (q_out, k_out)


def append(k_pages, v_pages, table, pos, k, v, seq=None, rotary=None, q=None, q_out=None):
    """Row r's keys (turned by `rotary`) and values [rows, n_kv_heads, head_dim]
    go to position pos[r] of sequence seq[r] (r without `seq`); its queries,
    turned, to q_out, which is returned.  A row without a page for its position
    (pos -1, say) is left out, its q_out too."""
    _detached(k, v, q, k_pages, v_pages, q_out)
    d, (n_pages, kv, ps, hd) = _pages(k_pages, v_pages, table)
    dev, dt = k_pages.device, k_pages.dtype
    rows = pos.shape[0]
    shape = (rows, kv, hd)
    a, o, heads = (None, 0, 0), (None, 0, 0), 0
    if q is not None:
        if q.dim() != 3:
            _refuse("queries are [rows, heads, head_dim]")
        heads = q.shape[1]
        qs = (rows, heads, hd)
        a = _heads(q, dev, dt, qs, "q")
        q_out, o = _out(q_out, q, qs, "q_out")
    b, c = _heads(k, dev, dt, shape, "k"), _heads(v, dev, dt, shape, "v")
    ts = table.shape
    tab = _ints(table, dev, ts, "table")
    p = _ints(pos, dev, (rows,), "pos")
    s = None if seq is None else _ints(seq, dev, (rows,), "seq")
    plan = None if rotary is None else _plan(rotary, dev, hd)
    if rows > 0:
        _run(dexlib.load().dex_pages_append, dev, d, hd, plan, rows, s, p, *a, heads, *o, *b, *c, kv, k_pages.data_ptr(),
             v_pages.data_ptr(), n_pages, ps, tab, ts[0], ts[1])
    return q_out


def attention(q, k_pages, v_pages, table, lens, seq=None, max_len=None, scale=None, window=0, group=1, out=None,
              return_lse=False):
    """Attention of one new token a row: q [rows, heads, head_dim] over the
    first lens[r] keys of sequence seq[r] (r without `seq`), the last `window`
    of them if that is not 0.  `max_len` bounds lens (the table's width
    otherwise): the tighter, the less work memory.  group: so many
    consecutive rows may share leading pages, which are then read once (of
    rows that have keys and begin at the same key; dex.h has the steps).
    Returns out, or (out, lse); a row without keys gets 0 and -inf."""
    _detached(q, k_pages, v_pages, out)
    d, (n_pages, kv, ps, hd) = _pages(k_pages, v_pages, table)
    dev, dt = k_pages.device, k_pages.dtype
    if q.dim() != 3:
        _refuse("queries are [rows, heads, head_dim]")
    rows, heads = q.shape[0], q.shape[1]
    shape = (rows, heads, hd)
    a = _heads(q, dev, dt, shape, "q")
    out, o = _out(out, q, shape, "out")
    ts = table.shape
    tab = _ints(table, dev, ts, "table")
    n = _ints(lens, dev, (rows,), "lens")
    s = None if seq is None else _ints(seq, dev, (rows,), "seq")
    most = ts[1] * ps
    if max_len is None or max_len > most:
        max_len = most
    if max_len < 0 or not 0 <= window < 1 << 31 or not 1 <= group < 1 << 31:
        _refuse("max_len or window is below 0, or group below 1, or past 2^31 - 1")
    lse = torch.empty((rows, heads), dtype=torch.float32, device=dev) if return_lse else None
    if rows > 0:
        size = _attention_work(rows, heads, kv, hd, max_len, group)
        work = torch.empty(size, dtype=torch.uint8, device=dev) if size else None
        _run(dexlib.load().dex_pages_attention, dev, d, hd, heads, kv, rows, s, n, max_len, window, group,
             1.0 / math.sqrt(hd) if scale is None else scale, *a, k_pages.data_ptr(), v_pages.data_ptr(), n_pages, ps, tab,
             ts[0], ts[1], *o, None if lse is None else lse.data_ptr(), None if work is None else work.data_ptr())
    return (out, lse) if return_lse else out


def _tables(table, ref, lens=None):
    if table.device.type != "cuda":
        _refuse("table is not on a GPU")
    if table.dim() != 2 or ref.dim() != 1:
        _refuse("table is [n_seqs, max_pages], ref is [n_pages]")
    dev = table.device
    p = [_ints(table, dev, table.shape, "table"), _ints(ref, dev, ref.shape, "ref")]
    if lens is not None:
        p.append(_ints(lens, dev, (table.shape[0],), "lens"))
    return dev, p


def fork(table, ref, lens, parent, out=None):
    """Sequence s becomes a copy of sequence parent[s] that shares its pages, or
    empty where parent[s] is no sequence; pages that nobody holds any more are
    free (ref 0).  Returns (table, ref, lens): `out`, new tensors without it;
    out=(table, ref, lens) works in place."""
    dev, p = _tables(table, ref, lens)
    if out is None:
        out = (torch.empty_like(table), torch.empty_like(ref), torch.empty_like(lens))
    n, c = table.shape
    _run(dexlib.load().dex_pages_fork, dev, *p, _ints(parent, dev, (n,), "parent"), n, c, ref.shape[0],
         _ints(out[0], dev, table.shape, "out[0]"), _ints(out[1], dev, ref.shape, "out[1]"),
         _ints(out[2], dev, lens.shape, "out[2]"))
    return out


class Reserved(NamedTuple):
    """What reserve granted: pos [n_seqs], the first new position of each
    sequence (-1: none), and the copies to make first (src, dst, tokens
    [n_seqs]; behind the last -1, -1, 0); state: copies, pages taken, pages
    missing, whether a sequence outgrows its table."""
    pos: torch.Tensor
    src: torch.Tensor
    dst: torch.Tensor
    tokens: torch.Tensor
    state: torch.Tensor

    def places(self, draft):
        """The positions [n_seqs, draft] of each sequence's `draft` tokens from pos
        on, as `append` takes them: all -1 where nothing was granted."""
        pos = self.pos[:, None]
        return torch.where(pos < 0, -1, pos + torch.arange(draft, dtype=torch.int32, device=pos.device))


def reserve(table, ref, lens, n_new, page_size):
    """Room for n_new[s] more tokens of every sequence, in place on table, ref
    and lens, with copies on write where a partly filled page is shared.  If
    the pages do not suffice nothing changes and every pos is -1."""
    dev, p = _tables(table, ref, lens)
    if not 1 <= page_size <= 1024:
        _refuse("page_size is not a power of two up to 1024")
    n, c = table.shape
    pn = _ints(n_new, dev, (n,), "n_new")
    buf = torch.empty(4 * n + 4, dtype=torch.int32, device=dev)
    got = Reserved(*buf.split((n, n, n, n, 4)))
    at = buf.data_ptr()
    _run(dexlib.load().dex_pages_reserve, dev, *p, pn, n, c, ref.shape[0], page_size, at, at + 4 * n, at + 8 * n,
         at + 12 * n, at + 16 * n)
    return got


class Compacted(NamedTuple):
    """new [n_pages]: each page's new number (-1: free); the moves for copy
    (src, dst [n_pages / 2], behind the last -1); state: moves, pages in use."""
    new: torch.Tensor
    src: torch.Tensor
    dst: torch.Tensor
    state: torch.Tensor


def compact(table, ref, out=None):
    """Renumbers the pages in use to the front.  out: (table, ref) to write to;
    without it both change in place.  `copy` has to move the contents before
    they are used again."""
    dev, p = _tables(table, ref)
    t, r = (table, ref) if out is None else out
    n, half = ref.shape[0], ref.shape[0] // 2
    buf = torch.empty(n + 2 * half + 4, dtype=torch.int32, device=dev)
    got = Compacted(*buf.split((n, half, half, 4)))
    at = buf.data_ptr()
    _run(dexlib.load().dex_pages_compact, dev, *p, table.shape[0], table.shape[1], n,
         _ints(t, dev, table.shape, "out[0]"), _ints(r, dev, ref.shape, "out[1]"), at, at + 4 * n, at + 4 * (n + half),
         at + 4 * (n + 2 * half))
    return got


def copy(k_pool, v_pool, src, dst, count=None, tokens=None):
    """Copies the pages dst[i] from src[i], i < count[0] (all without it), of
    every layer of the pools [n_layers, n_pages, n_kv_heads, page_size,
    head_dim]; with `tokens`, their first tokens[i] slots."""
    _detached(k_pool, v_pool)
    d = _gpu(k_pool, "k_pool")
    dev = k_pool.device
    if k_pool.dim() != 5 or not k_pool.is_contiguous():
        _refuse("pools are contiguous [n_layers, n_pages, n_kv_heads, page_size, head_dim]")
    if (v_pool.dtype is not k_pool.dtype or v_pool.device != dev or v_pool.shape != k_pool.shape
            or not v_pool.is_contiguous()):
        _refuse("values and keys differ in type, device or shape")
    layers, n_pages, kv, ps, hd = k_pool.shape
    n = src.shape[0]
    s, t = _ints(src, dev, (n,), "src"), _ints(dst, dev, (n,), "dst")
    tok = None if tokens is None else _ints(tokens, dev, (n,), "tokens")
    num = None
    if count is not None:
        if count.dim() != 1 or count.shape[0] < 1:
            _refuse("count holds the number of entries in its first element")
        num = _ints(count, dev, count.shape, "count")
    if n > 0:
        _run(dexlib.load().dex_pages_copy, dev, d, hd, layers, n_pages, kv, ps, k_pool.data_ptr(), v_pool.data_ptr(), s, t,
             tok, num, n)


def beam_select(logits, scores, n_out=None, done=None, eos=-1):
    """The n_out (beams by default) best continuations of each request: logits
    [requests * beams, vocab] (rows at any stride), scores [requests, beams]
    float32, done [requests, beams] bool.  Returns parent (rows of logits),
    token, score and done, [requests, n_out] each."""
    _detached(logits, scores)
    d = _gpu(logits, "logits")
    dev = logits.device
    if scores.dim() != 2 or scores.dtype is not torch.float32 or scores.device != dev or not scores.is_contiguous():
        _refuse("scores are contiguous float32 [requests, beams] on the logits' device")
    requests, beams = scores.shape
    if logits.dim() != 2 or logits.shape[0] != requests * beams or (logits.stride(1) != 1 and logits.shape[1] > 1):
        _refuse("logits are [requests * beams, vocab], a row's dense")
    vocab, ld = logits.shape[1], logits.stride(0)
    if done is not None and (done.dtype is not torch.bool or done.device != dev or done.shape != scores.shape
                             or not done.is_contiguous()):
        _refuse("done is a contiguous bool tensor like scores")
    n = beams if n_out is None else int(n_out)
    if not 1 <= n <= 64 or not -1 <= eos < vocab:
        _refuse("n_out is not 1 to 64, or eos not in [-1, vocab)")
    shape = (requests, n)
    score = torch.empty_like(scores) if n == beams else scores.new_empty(shape)
    parent = torch.empty_like(score, dtype=torch.int32)
    token, ends = torch.empty_like(parent), torch.empty_like(score, dtype=torch.bool)
    if requests > 0:
        work = torch.empty(_beam_work(d, requests, beams, vocab, n), dtype=torch.uint8, device=dev)
        _run(dexlib.load().dex_beam_select, dev, d, logits.data_ptr(), ld, requests, beams, vocab, scores.data_ptr(),
             None if done is None else done.data_ptr(), eos, n, parent.data_ptr(), token.data_ptr(), score.data_ptr(),
             ends.data_ptr(), work.data_ptr())
    return parent, token, score, ends


# ------------------------------------------ trees, chosen pages and eviction

_MAX_DRAFT = 256


@functools.lru_cache(maxsize=4096)
def _tree_work(*sizes):
    return dexlib.load().dex_pages_tree_attention_work(*sizes)


@functools.lru_cache(maxsize=4096)
def _sparse_work(*sizes):
    return dexlib.load().dex_pages_sparse_attention_work(*sizes)


@functools.lru_cache(maxsize=4096)
def _weigh_work(*sizes):
    return max(16, dexlib.load().dex_pages_weigh_work(*sizes))


def _bytes(n, device):
    return torch.empty(n, dtype=torch.uint8, device=device) if n else None


def _trees(parent):
    """Checks [n, draft] int32 on a GPU: device, n, draft."""
    if parent.device.type != "cuda":
        _refuse("parent is not on a GPU")
    if parent.dim() != 2 or not 1 <= parent.shape[1] <= _MAX_DRAFT:
        _refuse(f"parent is [n_trees, draft], draft 1 to {_MAX_DRAFT}")
    return parent.device, parent.shape[0], parent.shape[1]


def tree_mask(parent):
    """Trees of drafted tokens, parent [n, draft] int32: node i continues node
    parent[i] < i, or is a root (-1).  Returns mask [n, draft, words] int64, bit j
    of row i set if j is node i or an ancestor, and depth [n, draft] int32."""
    dev, n, t = _trees(parent)
    p = _ints(parent, dev, (n, t), "parent")
    mask = torch.empty((n, t, (t + 63) // 64), dtype=torch.int64, device=dev)
    depth = torch.empty_like(parent)
    if n > 0:
        _run(dexlib.load().dex_tree_mask, dev, p, n, t, mask.data_ptr(), depth.data_ptr())
    return mask, depth


def tree_accept(parent, token, target, n_draft=None, root=None):
    """The path of each tree that the model agrees with: node i is accepted if its
    parent is and token[i] == target[parent[i]] (all [n, draft] int32), a root if
    token[i] == root (root [n] int32; always without it); nodes from n_draft [n]
    on are none.  Returns path [n, draft] (nodes from a root to the deepest
    accepted one, then -1), count [n] and the next token [n]."""
    dev, n, t = _trees(parent)
    shape = (n, t)
    args = [_ints(x, dev, shape, name) for x, name in ((parent, "parent"), (token, "token"), (target, "target"))]
    nd = None if n_draft is None else _ints(n_draft, dev, (n,), "n_draft")
    r = None if root is None else _ints(root, dev, (n,), "root")
    path = torch.empty_like(parent)
    both = torch.empty((2, n), dtype=torch.int32, device=dev)
    if n > 0:
        at = both.data_ptr()
        _run(dexlib.load().dex_tree_accept, dev, *args, nd, r, n, t, path.data_ptr(), at, at + 4 * n)
    return path, both[0], both[1]


def _max_len(max_len, most):
    if max_len is None or max_len > most:
        return most
    if max_len < 0:
        _refuse("max_len is below 0")
    return max_len


def tree_attention(q, k_pages, v_pages, table, lens, mask, n_draft=None, seq=None, max_len=None, scale=None, out=None,
                   return_lse=False):
    """Attention of drafted tokens: q [n * draft, heads, head_dim], `draft` rows
    a tree, over the first lens[b] keys of sequence seq[b] (b without `seq`) and
    the drafted keys at positions lens[b] + j whose bit is set in mask[b, i]
    (`tree_mask`; any other mask works), j < n_draft[b].  `max_len` bounds lens.
    Returns out, or (out, lse); a row that sees nothing, and the rows from
    n_draft[b] on, get 0 and -inf."""
    _detached(q, k_pages, v_pages, out)
    d, (n_pages, kv, ps, hd) = _pages(k_pages, v_pages, table)
    dev, dt = k_pages.device, k_pages.dtype
    if q.dim() != 3:
        _refuse("queries are [n_trees * draft, heads, head_dim]")
    if mask.dim() != 3 or mask.dtype is not torch.int64 or mask.device != dev or not mask.is_contiguous():
        _refuse("mask is a contiguous int64 [n_trees, draft, words] tensor on the cache's device")
    n, t, words = mask.shape
    if not 1 <= t <= _MAX_DRAFT or words != (t + 63) // 64:
        _refuse(f"mask has 1 to {_MAX_DRAFT} drafted rows of ceil(draft / 64) words")
    heads = q.shape[1]
    shape = (n * t, heads, hd)
    a = _heads(q, dev, dt, shape, "q")
    out, o = _out(out, q, shape, "out")
    ts = table.shape
    tab = _ints(table, dev, ts, "table")
    length = _ints(lens, dev, (n,), "lens")
    nd = None if n_draft is None else _ints(n_draft, dev, (n,), "n_draft")
    s = None if seq is None else _ints(seq, dev, (n,), "seq")
    max_len = _max_len(max_len, ts[1] * ps)
    lse = torch.empty((n * t, heads), dtype=torch.float32, device=dev) if return_lse else None
    if n > 0:
        work = _bytes(_tree_work(d, n, t, heads, kv, hd, max_len), dev)
        _run(dexlib.load().dex_pages_tree_attention, dev, d, hd, heads, kv, n, t, s, length, nd, max_len,
             1.0 / math.sqrt(hd) if scale is None else scale, *a, mask.data_ptr(), k_pages.data_ptr(), v_pages.data_ptr(),
             n_pages, ps, tab, ts[0], ts[1], *o, None if lse is None else lse.data_ptr(),
             None if work is None else work.data_ptr())
    return (out, lse) if return_lse else out


def keep(k_pool, v_pool, table, index, count, first=None, to=None):
    """Position first[s] + j of sequence s receives keys and values of its
    position first[s] + index[j], j < count[s], in every layer of the pools
    [n_layers, n_pages, n_kv_heads, page_size, head_dim]; count and first (0
    without it) are [n_seqs] int32.  index is [n_seqs, n], the same for all, or
    [n_seqs, n_kv_heads, n], or [n_layers, n_seqs, n_kv_heads, n].  In place an
    entry with index[j] <= j copies nothing; `to` [n_seqs, pages] is another
    table to write to.  Pages written to have no other holder."""
    _detached(k_pool, v_pool)
    d = _gpu(k_pool, "k_pool")
    dev = k_pool.device
    if k_pool.dim() != 5 or not k_pool.is_contiguous():
        _refuse("pools are contiguous [n_layers, n_pages, n_kv_heads, page_size, head_dim]")
    if (v_pool.dtype is not k_pool.dtype or v_pool.device != dev or v_pool.shape != k_pool.shape
            or not v_pool.is_contiguous()):
        _refuse("values and keys differ in type, device or shape")
    layers, n_pages, kv, ps, hd = k_pool.shape
    if table.dim() != 2 or (to is not None and to.dim() != 2):
        _refuse("tables are [n_seqs, max_pages]")
    n = table.shape[0]
    lists = {2: (n,), 3: (n, kv), 4: (layers, n, kv)}.get(index.dim())
    if lists is None or tuple(index.shape[:-1]) != lists:
        _refuse("index is [n_seqs, n], [n_seqs, n_kv_heads, n] or [n_layers, n_seqs, n_kv_heads, n]")
    cap = index.shape[-1]
    at = _ints(index, dev, index.shape, "index")
    many = kv if index.dim() > 2 else 1
    strides = (n * many * cap if index.dim() == 4 else 0, many * cap, cap if many > 1 else 0)
    c = _ints(count, dev, (n,), "count")
    f = None if first is None else _ints(first, dev, (n,), "first")
    tab = _ints(table, dev, table.shape, "table")
    other, width = (None, 0) if to is None else (_ints(to, dev, (n, to.shape[1]), "to"), to.shape[1])
    if n > 0 and cap > 0:
        _run(dexlib.load().dex_pages_keep, dev, d, hd, layers, n_pages, kv, ps, k_pool.data_ptr(), v_pool.data_ptr(), tab, n,
             table.shape[1], other, width, f, at, *strides, cap, c)


def trim(table, ref, lens, page_size, out=None):
    """Pages behind the sequences' last tokens (lens) leave the table and lose a
    holder.  out: (table, ref) to write to; without it both change in place.
    Returns them."""
    dev, p = _tables(table, ref, lens)
    if not 1 <= page_size <= 1024:
        _refuse("page_size is not a power of two up to 1024")
    t, r = (table, ref) if out is None else out
    _run(dexlib.load().dex_pages_trim, dev, *p, table.shape[0], table.shape[1], ref.shape[0], page_size,
         _ints(t, dev, table.shape, "out[0]"), _ints(r, dev, ref.shape, "out[1]"))
    return t, r


def _bounds(bounds, k_dtype, dev, shape, name="bounds"):
    if bounds.dtype is not k_dtype or bounds.device != dev or bounds.shape != shape or not bounds.is_contiguous():
        _refuse(f"{name}: a contiguous {k_dtype} tensor of shape {tuple(shape)} on {dev} is wanted")
    return bounds.data_ptr()


def page_bounds(k_pages, table, lens, n_new=None, out=None):
    """The least and the largest key of each page in every dimension, [n_pages,
    n_kv_heads, 2, head_dim]: those of the pages that hold the last n_new (all
    without it) of lens[s] tokens of the sequences, in `out` (0 elsewhere in a
    new one)."""
    _detached(k_pages, out)
    d, (n_pages, kv, ps, hd) = _pages(k_pages, k_pages, table)
    dev = k_pages.device
    shape = (n_pages, kv, 2, hd)
    out = k_pages.new_zeros(shape) if out is None else out
    at = _bounds(out, k_pages.dtype, dev, shape, "out")
    ts = table.shape
    tab, length = _ints(table, dev, ts, "table"), _ints(lens, dev, (ts[0],), "lens")
    n_new = _max_len(n_new, ts[1] * ps)
    if ts[0] > 0:
        _run(dexlib.load().dex_pages_bounds, dev, d, hd, k_pages.data_ptr(), n_pages, kv, ps, tab, ts[0], ts[1], length, n_new,
             at)
    return out


def select_pages(q, bounds, table, lens, page_size, n_select, sinks=1, recent=1, seq=None, max_len=None):
    """The pages to read for each row and kv head: q [rows, heads, head_dim],
    bounds as `page_bounds` gives them.  Of the table's columns that hold tokens,
    the first `sinks`, the last `recent` and those whose bounds allow the largest
    products with the kv head's queries, n_select in all.  Returns columns [rows,
    n_kv_heads, n_select] int32, ascending, then -1."""
    _detached(q, bounds)
    d = _gpu(bounds, "bounds")
    dev, dt = bounds.device, bounds.dtype
    if bounds.dim() != 4 or bounds.shape[2] != 2 or not bounds.is_contiguous():
        _refuse("bounds are contiguous [n_pages, n_kv_heads, 2, head_dim]")
    n_pages, kv, _, hd = bounds.shape
    if q.dim() != 3 or table.dim() != 2:
        _refuse("queries are [rows, heads, head_dim], table is [n_seqs, max_pages]")
    rows, heads = q.shape[:2]
    a = _heads(q, dev, dt, (rows, heads, hd), "q")
    ts = table.shape
    tab, length = _ints(table, dev, ts, "table"), _ints(lens, dev, (rows,), "lens")
    s = None if seq is None else _ints(seq, dev, (rows,), "seq")
    if not 1 <= page_size <= 1024:
        _refuse("page_size is not a power of two up to 1024")
    max_len = _max_len(max_len, ts[1] * page_size)
    if not 1 <= n_select < 1 << 31 or not 0 <= sinks <= n_select or not 0 <= recent <= n_select:
        _refuse("n_select is below 1 or below sinks + recent")
    columns = torch.empty((rows, kv, n_select), dtype=torch.int32, device=dev)
    if rows > 0:
        work = torch.empty(rows * kv * -(-max_len // page_size), dtype=torch.int64, device=dev)
        _run(dexlib.load().dex_pages_select, dev, d, hd, heads, kv, rows, s, length, max_len, *a, bounds.data_ptr(), n_pages,
             page_size, tab, ts[0], ts[1], n_select, sinks, recent, columns.data_ptr(), work.data_ptr())
    return columns


def sparse_attention(q, k_pages, v_pages, table, lens, columns, seq=None, scale=None, out=None, return_lse=False):
    """`attention` over the tokens of the listed columns of the table alone,
    columns [rows, n_kv_heads, n] int32 as `select_pages` gives them."""
    _detached(q, k_pages, v_pages, out)
    d, (n_pages, kv, ps, hd) = _pages(k_pages, v_pages, table)
    dev, dt = k_pages.device, k_pages.dtype
    if q.dim() != 3 or columns.dim() != 3:
        _refuse("queries are [rows, heads, head_dim], columns [rows, n_kv_heads, n]")
    rows, heads = q.shape[:2]
    shape = (rows, heads, hd)
    a = _heads(q, dev, dt, shape, "q")
    out, o = _out(out, q, shape, "out")
    ts, n = table.shape, columns.shape[2]
    tab, length = _ints(table, dev, ts, "table"), _ints(lens, dev, (rows,), "lens")
    c = _ints(columns, dev, (rows, kv, n), "columns")
    s = None if seq is None else _ints(seq, dev, (rows,), "seq")
    lse = torch.empty((rows, heads), dtype=torch.float32, device=dev) if return_lse else None
    if rows > 0:
        work = _bytes(_sparse_work(d, rows, heads, kv, hd, n, ps), dev)
        _run(dexlib.load().dex_pages_sparse_attention, dev, d, hd, heads, kv, rows, s, length,
             1.0 / math.sqrt(hd) if scale is None else scale, *a, c, n, k_pages.data_ptr(), v_pages.data_ptr(), n_pages, ps,
             tab, ts[0], ts[1], *o, None if lse is None else lse.data_ptr(), None if work is None else work.data_ptr())
    return (out, lse) if return_lse else out


def _weights(t, dev, rows, kv, name):
    """[rows, n_kv_heads, n] float32, contiguous: its address."""
    if (t.dtype is not torch.float32 or t.device != dev or t.dim() != 3 or t.shape[:2] != (rows, kv)
            or not t.is_contiguous()):
        _refuse(f"{name} is a contiguous float32 [{rows}, {kv}, n] tensor on {dev}")
    return t.data_ptr()


def weigh(q, k_pages, v_pages, table, lens, weight, weight_out=None, seq=None, max_len=None, scale=None, out=None,
          return_lse=False):
    """`attention` of one new token a row that also adds up what each key was
    given: weight_out[r, h, j] = weight[r, h, j] + the softmax weights of key j <
    lens[r], summed over the query heads of kv head h; float32 [rows, n_kv_heads,
    n], n at least max_len.  Without weight_out in place; what lies behind
    lens[r] stays.  Returns out, or (out, lse)."""
    _detached(q, k_pages, v_pages, weight, weight_out, out)
    d, (n_pages, kv, ps, hd) = _pages(k_pages, v_pages, table)
    dev, dt = k_pages.device, k_pages.dtype
    if q.dim() != 3:
        _refuse("queries are [rows, heads, head_dim]")
    rows, heads = q.shape[:2]
    shape = (rows, heads, hd)
    a = _heads(q, dev, dt, shape, "q")
    out, o = _out(out, q, shape, "out")
    ts = table.shape
    tab, length = _ints(table, dev, ts, "table"), _ints(lens, dev, (rows,), "lens")
    s = None if seq is None else _ints(seq, dev, (rows,), "seq")
    max_len = _max_len(max_len, ts[1] * ps)
    w = _weights(weight, dev, rows, kv, "weight")
    to, wo = (weight, w) if weight_out is None else (weight_out, _weights(weight_out, dev, rows, kv, "weight_out"))
    if min(weight.shape[2], to.shape[2]) < max_len:
        _refuse("the weights have fewer columns than max_len")
    lse = torch.empty((rows, heads), dtype=torch.float32, device=dev) if return_lse else None
    if rows > 0:
        work = _bytes(_weigh_work(d, rows, heads, kv, hd, max_len), dev)
        _run(dexlib.load().dex_pages_weigh, dev, d, hd, heads, kv, rows, s, length, max_len,
             1.0 / math.sqrt(hd) if scale is None else scale, *a, w, weight.shape[2], wo, to.shape[2], k_pages.data_ptr(),
             v_pages.data_ptr(), n_pages, ps, tab, ts[0], ts[1], *o, None if lse is None else lse.data_ptr(), work.data_ptr())
    return (out, lse) if return_lse else out


def evict(weight, lens, budget, sinks=0, recent=1, weight_out=None):
    """Which keys of each sequence and kv head stay, by their accumulated weight
    [n_seqs, n_kv_heads, n] float32: the first `sinks`, the last `recent` and the
    heaviest others, min(lens[s], n, budget) in all (keys from n on, which have no
    weight, do not stay).  Returns index [n_seqs, n_kv_heads, budget] int32,
    ascending, then -1, as `keep` takes it, and count [n_seqs], the sequences' new
    lengths; weight_out (`weight` without it) receives the kept keys' weights,
    then 0."""
    _detached(weight, weight_out)
    if weight.device.type != "cuda":
        _refuse("weight is not on a GPU")
    dev = weight.device
    if weight.dim() != 3:
        _refuse("weight is [n_seqs, n_kv_heads, n]")
    n, kv, cap = weight.shape
    w = _weights(weight, dev, n, kv, "weight")
    to = weight if weight_out is None else weight_out
    wo = _weights(to, dev, n, kv, "weight_out")
    if to.shape != weight.shape:
        _refuse("weight_out has another shape than weight")
    length = _ints(lens, dev, (n,), "lens")
    if not 1 <= budget < 1 << 31 or not 0 <= sinks <= budget or not 0 <= recent <= budget:
        _refuse("budget is below 1 or below sinks + recent")
    index = torch.empty((n, kv, budget), dtype=torch.int32, device=dev)
    count = torch.empty(n, dtype=torch.int32, device=dev)
    if n > 0:
        _run(dexlib.load().dex_pages_evict, dev, w, cap, n, kv, cap, length, budget, sinks, recent, index.data_ptr(),
             count.data_ptr(), wo, cap)
    return index, count



class PagedCache:
    """Keys and values of every layer in pages, with the page table, the
    holders' counts and the lengths of n_seqs sequences, all free at first; with
    `bounds` each layer's page bounds too."""

    def __init__(self, n_layers, n_kv_heads, head_dim, page_size, n_pages, n_seqs, max_pages, dtype=torch.bfloat16,
                 device="cuda", bounds=False):
        shape = (n_layers, n_pages, n_kv_heads, page_size, head_dim)
        self.k = torch.zeros(shape, dtype=dtype, device=device)
        self.v = torch.zeros(shape, dtype=dtype, device=device)
        self.table = torch.full((n_seqs, max_pages), -1, dtype=torch.int32, device=device)
        self.ref = torch.zeros(n_pages, dtype=torch.int32, device=device)
        self.lens = torch.zeros(n_seqs, dtype=torch.int32, device=device)
        # with `bounds`: each layer's, for attention over chosen pages
        self.bounds = torch.zeros((n_layers, n_pages, n_kv_heads, 2, head_dim), dtype=dtype, device=device) if bounds else None
        self.n_layers, self.page_size = n_layers, page_size
        self._copies = False                      # whether `copy` is known to take these pools

    def _check_copy(self):
        """Refuses what `copy` would refuse, before a table changes."""
        _detached(self.k, self.v)
        if not self._copies:                      # of no entries: the sizes are looked at, nothing is launched
            layers, n_pages, kv, ps, hd = self.k.shape
            _run(dexlib.load().dex_pages_copy, self.k.device, _gpu(self.k, "k"), hd, layers, n_pages, kv, ps,
                 self.k.data_ptr(), self.v.data_ptr(), None, None, None, None, 0)
            self._copies = True

    def reserve(self, n_new):
        """Room for n_new [n_seqs] tokens, shared pages copied: the Reserved."""
        self._check_copy()
        got = reserve(self.table, self.ref, self.lens, n_new, self.page_size)
        copy(self.k, self.v, got.src, got.dst, got.state, got.tokens)
        return got

    def append(self, layer, pos, q, k, v, rotary=None, seq=None):
        """Writes a layer's keys and values at `pos`; the queries, turned."""
        return append(self.k[layer], self.v[layer], self.table, pos, k, v, seq=seq, rotary=rotary, q=q)

    def attention(self, layer, q, lens=None, seq=None, **kw):
        """Attention over a layer, by default of row r over all of sequence r."""
        return attention(q, self.k[layer], self.v[layer], self.table, self.lens if lens is None else lens, seq=seq, **kw)

    def fork(self, parent):
        """Sequence s goes on from sequence parent[s] (-1: is freed)."""
        fork(self.table, self.ref, self.lens, parent, out=(self.table, self.ref, self.lens))

    def compact(self):
        """Moves the pages in use to the front: the Compacted."""
        self._check_copy()
        got = compact(self.table, self.ref)
        copy(self.k, self.v, got.src, got.dst, got.state)
        return got

    def tree_attention(self, layer, q, lens, mask, **kw):
        """Attention of drafted tokens over a layer; lens: the sequences' tokens
        before their trees."""
        return tree_attention(q, self.k[layer], self.v[layer], self.table, lens, mask, **kw)

    def accept(self, lens, path, count):
        """Of the tokens that each sequence holds from lens [n_seqs] on (its length
        before `reserve`), those of the path stay, behind the sequence; the rest and
        their pages are given back.  path and count as `tree_accept` gives them for
        the trees' tokens that were granted (n_draft); a sequence without any stays
        as it is."""
        count = torch.minimum(count, self.lens - lens)
        keep(self.k, self.v, self.table, path, count, first=lens)
        torch.add(lens, count, out=self.lens)
        trim(self.table, self.ref, self.lens, self.page_size)

    def update_bounds(self, layer, n_new=None):
        """The bounds of the pages that hold the last n_new tokens (all without
        it); after `fork`, `reserve` and `append` those of the new tokens, after
        `accept` those of the accepted ones, which have moved (n_new as many as a
        path has at most), after `compact` or `evict` all."""
        if self.bounds is None:
            _refuse("the cache keeps no bounds (bounds=True)")
        page_bounds(self.k[layer], self.table, self.lens, n_new=n_new, out=self.bounds[layer])

    def _row_lens(self, lens, seq):
        """The rows' lengths: by default row r is sequence r, over all its tokens."""
        if lens is None and seq is not None:
            _refuse("rows of other sequences (seq) go with their lengths (lens)")
        return self.lens if lens is None else lens

    def sparse_attention(self, layer, q, n_select, sinks=1, recent=1, lens=None, seq=None, max_len=None, **kw):
        """Attention of row r over the n_select pages of sequence r that its query
        selects (`update_bounds` has to have seen its tokens); with seq [rows] over
        those of sequence seq[r], whose first lens[r] keys it sees.  `max_len` bounds
        the lengths: the tighter, the fewer pages are looked at."""
        if self.bounds is None:
            _refuse("the cache keeps no bounds (bounds=True)")
        lens = self._row_lens(lens, seq)
        columns = select_pages(q, self.bounds[layer], self.table, lens, self.page_size, n_select, sinks=sinks, recent=recent,
                               seq=seq, max_len=max_len)
        return sparse_attention(q, self.k[layer], self.v[layer], self.table, lens, columns, seq=seq, **kw)

    def weigh(self, layer, q, weight, lens=None, seq=None, **kw):
        """Attention of row r over sequence r that adds its weights to weight[r];
        with seq [rows] over the first lens[r] keys of sequence seq[r]."""
        lens = self._row_lens(lens, seq)
        return weigh(q, self.k[layer], self.v[layer], self.table, lens, weight, seq=seq, **kw)

    def evict(self, weight, budget, sinks=0, recent=1, max_len=None):
        """Cuts every sequence to its `budget` heaviest keys (see `evict`), in place,
        by weight [n_layers, n_seqs, n_kv_heads, n], which is cut with it; n is at
        least max_len, which bounds the sequences' lengths (the table's width
        without it).  The sequences' pages have no other holders.  The keys keep the
        rotary positions that they have, and new tokens need positions of the
        caller's own count."""
        if weight.dim() != 4 or weight.shape[:3] != (self.n_layers, len(self.lens), self.k.shape[2]):
            _refuse("weight is [n_layers, n_seqs, n_kv_heads, n]")
        if not weight.is_contiguous():            # (flattened it would be a copy, and only that be cut)
            _refuse("weight is not contiguous")
        if weight.shape[3] < _max_len(max_len, self.table.shape[1] * self.page_size):
            _refuse("the weights have fewer columns than max_len")
        self._check_copy()
        n = len(self.lens)
        index, count = evict(weight.flatten(0, 1), self.lens.repeat(self.n_layers), budget, sinks=sinks, recent=recent)
        keep(self.k, self.v, self.table, index.unflatten(0, (self.n_layers, n)), count[:n])
        self.lens.copy_(count[:n])
        trim(self.table, self.ref, self.lens, self.page_size)
