"""Performance cases of the operators over a paged key/value cache.

What a serving loop with branches does between a model's matrix products, in
the order it does it:
  rope, append  rotary positions of queries and keys, alone or with the keys
                and values written into the cache's pages in the same launch;
  attention     one new token a row over the row's pages;
  beam          the best continuations over beams and vocabulary;
  step          the beams' page tables follow their parents, pages nobody holds
                are freed, every sequence gets room for its next token, and
                pages that several would write are copied first;
  compact       the pages in use move to the front of the cache.

Every kind has its plain form here (elementary torch operations, a whole batch
at a time) and the call of the framework's own operator.  Shapes are those of
the framework's models (32 / 8 heads of 128, 12 heads of 64, 4 of 32;
vocabulary 32000) or generic.
"""

from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ the cases

def _rope(rows, heads, kv_heads, head_dim, rot_dim, interleaved, dtype, scaling, first, spread, inverse=False):
    return {"kind": "rope", "rows": rows, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim,
            "rot_dim": rot_dim, "interleaved": interleaved, "dtype": dtype, "scaling": scaling, "first": first,
            "spread": spread, "inverse": inverse}


def _append(seqs, tokens, heads, kv_heads, head_dim, rot_dim, interleaved, dtype, scaling, page, first):
    return {"kind": "append", "seqs": seqs, "tokens": tokens, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rot_dim": rot_dim, "interleaved": interleaved, "dtype": dtype,
            "scaling": scaling, "page": page, "first": first}


def _attention(rows, shortest, longest, heads, kv_heads, head_dim, page, dtype, group=1, shared=0, window=0, empty=0):
    return {"kind": "attention", "rows": rows, "shortest": shortest, "longest": longest, "heads": heads,
            "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "dtype": dtype, "group": group,
            "shared": shared, "window": window, "empty": empty}


def _step(requests, beams, longest, page, layers, kv_heads, head_dim, dtype):
    return {"kind": "step", "requests": requests, "beams": beams, "longest": longest, "page": page,
            "layers": layers, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype}


def _compact(seqs, pages, moved, page, layers, kv_heads, head_dim, dtype):
    return {"kind": "compact", "seqs": seqs, "pages": pages, "moved": moved, "page": page, "layers": layers,
            "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype}


def _beam(requests, beams, vocab, dtype, finished, masked):
    return {"kind": "beam", "requests": requests, "beams": beams, "vocab": vocab, "dtype": dtype,
            "finished": finished, "masked": masked}


def listed():
    return [
        # queries and keys of a few rows at far positions, fp32: interleaved pairs, half of each head,
        # frequencies scaled band by band for a long context
        dict(_rope(77, 12, 12, 64, 32, True, "f32", "bands", 900000, 1000), name="rope_far_77"),
        # one decode step of four sequences: the smallest call, where latency counts
        dict(_append(4, 1, 32, 8, 128, 128, False, "bf16", "none", 16, 517), name="append_decode_4"),
        # eight prompts of 1024 tokens written into the cache
        dict(_append(8, 1024, 32, 8, 128, 128, False, "bf16", "linear", 64, 0), name="append_prompt_8x1024"),
        # one short request
        dict(_attention(1, 700, 700, 32, 8, 128, 16, "bf16"), name="attention_1x700"),
        # eight long documents
        dict(_attention(8, 8300, 8300, 32, 8, 128, 64, "bf16"), name="attention_8x8300"),
        # a serving batch: ragged lengths from one token to 16000, an empty row
        dict(_attention(64, 1, 16000, 32, 8, 128, 16, "bf16", empty=1), name="attention_64_ragged"),
        # sixteen requests of eight beams that share their prompt's pages
        dict(_attention(128, 4090, 4090, 32, 8, 128, 16, "bf16", group=8, shared=4000), name="attention_beams_16x8"),
        # an fp32 model with as many key heads as query heads, a sliding window
        dict(_attention(24, 50, 5000, 12, 12, 64, 32, "f32", window=2000), name="attention_f32_24"),
        # one decoding step's bookkeeping for eight requests of eight beams, all 32 layers' pages
        dict(_step(8, 8, 900, 16, 32, 8, 128, "bf16"), name="step_8x8"),
        # a small model's pool, half empty, compacted
        dict(_compact(32, 4096, 1000, 16, 12, 12, 64, "bf16"), name="compact_4096"),
        # one request with four beams
        dict(_beam(1, 4, 32000, "f32", 0, False), name="beam_1x4"),
        # 64 requests of eight beams, an odd vocabulary, some beams finished, part of the vocabulary masked
        dict(_beam(64, 8, 65537, "bf16", 3, True), name="beam_64x8_odd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "append", "attention", "attention", "attention", "step", "compact", "beam", "beam"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    heads, kv_heads, head_dim = rng.choice(((32, 8, 128), (32, 8, 128), (12, 12, 64), (4, 4, 32), (16, 2, 64),
                                            (28, 4, 128), (10, 5, 128)))
    page = rng.choice((8, 16, 16, 32, 64, 128))
    rot_dim = rng.choice((head_dim, head_dim, head_dim // 2, head_dim // 4))
    scaling = rng.choice(("none", "linear", "base", "bands"))
    interleaved = rng.random() < 0.5
    if kind == "rope":
        return _rope(_log_int(rng, 1, 8192), heads, kv_heads, head_dim, rot_dim, interleaved, dtype, scaling,
                     _log_int(rng, 1, 1 << 20), _log_int(rng, 8, 8192), rng.random() < 0.3)
    if kind == "append":
        seqs = _log_int(rng, 1, 64)
        tokens = 1 if rng.random() < 0.5 else _log_int(rng, 1, 8192 // seqs)
        return _append(seqs, tokens, heads, kv_heads, head_dim, rot_dim, interleaved, dtype, scaling, page,
                       _log_int(rng, 1, 3000))
    if kind == "attention":
        group = rng.choice((1, 1, 2, 4, 8))
        rows = group * _log_int(rng, 1, 64 // group)
        longest = _log_int(rng, 1, 16000)
        per_key = kv_heads * head_dim * (2 if dtype == "bf16" else 4)
        while rows > group and rows * longest * per_key > 1 << 29:
            rows -= group
        shared = longest * rng.randint(0, 9) // 10 if group > 1 else 0
        shortest = longest if group > 1 else rng.randint(1, longest)
        return _attention(rows, shortest, longest, heads, kv_heads, head_dim, page, dtype, group, shared,
                          rng.choice((0, 0, _log_int(rng, 16, 4096))), rng.choice((0, 0, 1)) if rows > 4 else 0)
    if kind == "step":
        beams = rng.choice((2, 3, 4, 5, 8))
        return _step(_log_int(rng, 1, 64 // beams), beams, _log_int(rng, 8, 900), page, rng.choice((2, 4, 12)),
                     kv_heads, head_dim, dtype)
    if kind == "compact":
        pages = _log_int(rng, 32, 2048)
        per_page = page * kv_heads * head_dim * (2 if dtype == "bf16" else 4)
        layers = max(1, min(12, (1 << 30) // (pages * per_page)))
        return _compact(rng.randint(1, 16), pages, rng.randint(1, pages // 4), page, layers, kv_heads, head_dim, dtype)
    beams = rng.choice((1, 2, 3, 4, 5, 8, 16))
    return _beam(_log_int(rng, 1, 256 // beams), beams, _log_int(rng, 500, 65000), dtype,
                 rng.choice((0, 1)) if beams > 1 else 0, rng.random() < 0.3)


# ------------------------------------------------- what a case's sizes come to

SCALING = {  # what a rotary plan is told; `slow` and `fast` are turns over the original context
    "none": dict(scaling=None),
    "linear": dict(scaling="linear", factor=4.0),
    "base": dict(scaling="base", factor=8.0),
    "bands": dict(scaling="bands", factor=16.0, original=8192, slow=1.0, fast=32.0,
                  amplitude=0.1 * math.log(16.0) + 1.0),
}
THETA = 1e4


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def _lengths(case):
    """The keys of every row: spread evenly over the logarithm of the range, `empty` rows of none."""
    n = case["rows"] // case["group"]
    lo, hi = case["shortest"], case["longest"]
    lens = [int(round(math.exp(math.log(lo) + (math.log(hi) - math.log(lo)) * (i / max(1, n - 1))))) for i in range(n)]
    lens[-1] = hi
    lens = [0 if i < case["empty"] else v for i, v in enumerate(lens)]
    return [v for v in lens for _ in range(case["group"])]


def _step_lengths(case):
    """The length of each request's beams: odd ones, none at a page's edge."""
    out = []
    for r in range(case["requests"]):
        v = max(3, case["longest"] - 37 * r % max(1, case["longest"] // 2))
        out.append(v + 1 if v % case["page"] == 0 else v)
    return out


def _children(beams):
    """How many of the next beams continue each of a request's beams."""
    c = [0] * beams
    left = beams
    for i in range(beams):
        c[i] = min(left, left // 2 + 1)
        left -= c[i]
    return c


def work(case):
    e = _elem(case)
    kind = case["kind"]
    if kind == "rope":
        n = case["rows"] * (case["heads"] + case["kv_heads"])
        return {"bytes": 2 * n * case["head_dim"] * e + 4 * case["rows"], "flops": 3 * n * case["rot_dim"]}
    if kind == "append":
        rows = case["seqs"] * case["tokens"]
        n = rows * (case["heads"] + 2 * case["kv_heads"])
        return {"bytes": 2 * n * case["head_dim"] * e + 8 * rows,
                "flops": 3 * rows * (case["heads"] + case["kv_heads"]) * case["rot_dim"]}
    if kind == "attention":
        lens = _lengths(case)
        seen = [min(v, case["window"]) if case["window"] else v for v in lens]
        g, ps = case["group"], case["page"]
        shared = case["shared"] // ps * ps
        keys = 0
        for r, (n, s) in enumerate(zip(lens, seen)):   # keys on a request's shared pages count once
            twice = max(0, min(n, shared) - (n - s)) if r % g else 0
            keys += s - twice
        io = case["rows"] * case["heads"] * (2 * case["head_dim"] * e + 4)
        return {"bytes": 2 * keys * case["kv_heads"] * case["head_dim"] * e + io + 4 * sum(-(-s // ps) for s in seen),
                "flops": 4 * sum(seen) * case["heads"] * case["head_dim"]}
    if kind == "step":
        rows, ps = case["requests"] * case["beams"], case["page"]
        lens = _step_lengths(case)
        width = max(lens) // ps + 2
        copies = sum(c - 1 for c in _children(case["beams"]) if c)
        slot = case["kv_heads"] * case["head_dim"] * e * 2 * case["layers"]
        return {"bytes": 8 * rows * width + 8 * _step_pages(case) + 2 * copies * slot * sum(v % ps for v in lens),
                "flops": 0}
    if kind == "compact":
        slot = case["kv_heads"] * case["head_dim"] * e * 2 * case["layers"] * case["page"]
        return {"bytes": 2 * case["moved"] * slot + 12 * case["pages"] + 4 * case["pages"], "flops": 0}
    n = case["requests"] * case["beams"]
    finished = case["requests"] * case["finished"]
    return {"bytes": (n - finished) * case["vocab"] * e + 20 * n, "flops": 4 * (n - finished) * case["vocab"]}


def _step_pages(case):
    """Pages of the pool of a step: what the sequences hold at most, and as many to take as they can need."""
    ps, b = case["page"], case["beams"]
    return sum(v // ps + b * (2 + 2) for v in _step_lengths(case)) + 8


# ------------------------------------------------------------- inputs on the GPU

def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if dtype == torch.float32 else dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    dtype = DTYPES[case["dtype"]]
    st = {"case": case, "kind": case["kind"]}

    def ints(a):
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()

    def rotary():
        # the plan a program makes once for its model
        if own:
            from paper_2606_29223_amd import paged
            st["rotary"] = paged.Rotary(case["head_dim"], rot_dim=case["rot_dim"], theta=THETA,
                                        interleaved=case["interleaved"], **SCALING[case["scaling"]])

    if case["kind"] == "rope":
        # queries and keys as a fused projection leaves them: rows of all heads, strided views
        h, kv, hd = case["heads"], case["kv_heads"], case["head_dim"]
        x = _normal(g, (case["rows"], h + 2 * kv, hd), dtype)
        st.update(q=x[:, :h], k=x[:, h:h + kv],
                  pos=ints(case["first"] + rng.integers(0, case["spread"], case["rows"])))
        rotary()
    elif case["kind"] == "append":
        h, kv, hd, ps = case["heads"], case["kv_heads"], case["head_dim"], case["page"]
        seqs, tokens = case["seqs"], case["tokens"]
        first = rng.integers(max(0, case["first"] // 2), case["first"] + 1, seqs)
        width = int((first.max() + tokens + ps - 1) // ps) + 1
        # a table whose pages past a sequence's end are absent; only the pages written to exist
        lo, hi = first // ps, (first + tokens - 1) // ps
        n_pages = seqs * (-(-tokens // ps) + 1) + 3
        ids = rng.permutation(n_pages)
        table = np.full((seqs, width), -1)
        at = 0
        for s in range(seqs):
            n = int(hi[s] - lo[s]) + 1
            table[s, lo[s]:hi[s] + 1] = ids[at:at + n]
            at += n
        x = _normal(g, (seqs * tokens, h + 2 * kv, hd), dtype)
        st.update(q=x[:, :h], k=x[:, h:h + kv], v=x[:, h + kv:], table=ints(table),
                  seq=ints(np.repeat(np.arange(seqs), tokens)),
                  pos=ints((first[:, None] + np.arange(tokens)[None]).reshape(-1)),
                  k_pages=_normal(g, (n_pages, kv, ps, hd), dtype), v_pages=_normal(g, (n_pages, kv, ps, hd), dtype))
        rotary()
    elif case["kind"] == "attention":
        kv, hd, ps, grp = case["kv_heads"], case["head_dim"], case["page"], case["group"]
        lens = np.array(_lengths(case)).reshape(-1, grp)
        lens = lens[rng.permutation(len(lens))].reshape(-1)
        rows = case["rows"]
        width = max(1, -(-int(lens.max()) // ps))
        shared = case["shared"] // ps
        need = sum(-(-int(v) // ps) for v in lens)
        ids = rng.permutation(need + 5)
        table = np.full((rows, width), -1)
        at = 0
        for r in range(rows):
            n = -(-int(lens[r]) // ps)
            k = min(shared, n) if r % grp else 0
            table[r, :k] = table[r - r % grp, :k]
            table[r, k:n] = ids[at:at + n - k]
            at += n - k
        n_pages = at + 5
        table[table >= 0] = rng.permutation(n_pages)[np.unique(table[table >= 0], return_inverse=True)[1]]
        st.update(q=2 * _normal(g, (rows, case["heads"], hd), dtype), table=ints(table), lens=ints(lens),
                  longest=int(lens.max()), k_pages=_normal(g, (n_pages, kv, ps, hd), dtype),
                  v_pages=_normal(g, (n_pages, kv, ps, hd), dtype))
    elif case["kind"] == "step":
        ps, b = case["page"], case["beams"]
        lens = _step_lengths(case)
        rows, width, n_pages = len(lens) * b, max(lens) // ps + 2, _step_pages(case)
        ids = rng.permutation(n_pages)
        table, parent, at = np.full((rows, width), -1), np.zeros(rows, np.int64), 0
        for r, n in enumerate(lens):
            full = max(0, n // ps - 1)          # pages the request's beams share; the last ones are each beam's own
            table[r * b:(r + 1) * b, :full] = ids[at:at + full]
            at += full
            for i in range(b):
                own_pages = n // ps + 1 - full
                table[r * b + i, full:full + own_pages] = ids[at:at + own_pages]
                at += own_pages
            parent[r * b:(r + 1) * b] = r * b + rng.permutation(np.repeat(rng.permutation(b), _children(b)))
        ref = np.bincount(table[table >= 0], minlength=n_pages)
        shape = (case["layers"], n_pages, case["kv_heads"], ps, case["head_dim"])
        st.update(table=ints(table), ref=ints(ref), lens=ints(np.repeat(lens, b)), parent=ints(parent),
                  n_new=ints(np.ones(rows)), page=ps, k_pool=_normal(g, shape, dtype), v_pool=_normal(g, shape, dtype))
        # where a program keeps the tables of its next step
        st["next"] = tuple(torch.empty_like(st[n]) for n in ("table", "ref", "lens"))
    elif case["kind"] == "compact":
        n, ps, seqs = case["pages"], case["page"], case["seqs"]
        live = n // 2
        used = np.concatenate([rng.permutation(live)[:live - case["moved"]],
                               live + rng.permutation(n - live)[:case["moved"]]])
        used = rng.permutation(used)
        width = -(-live // seqs) + 1
        table = np.full((seqs, width), -1)
        for s in range(seqs):                   # the sequences hold the pages in turn, and share the first
            mine = np.concatenate([used[:1], used[1 + s::seqs]])
            table[s, :len(mine)] = mine
        ref = np.bincount(table[table >= 0], minlength=n)
        shape = (case["layers"], n, case["kv_heads"], ps, case["head_dim"])
        st.update(table=ints(table), ref=ints(ref), k_pool=_normal(g, shape, dtype), v_pool=_normal(g, shape, dtype))
        st["next"] = tuple(torch.empty_like(st[n]) for n in ("table", "ref"))
    else:
        r, b, v = case["requests"], case["beams"], case["vocab"]
        logits = 3 * _normal(g, (r * b, v), dtype)
        if case["masked"]:                      # a grammar: two thirds of the vocabulary are not allowed
            logits.masked_fill_(torch.rand((1, v), generator=g, device="cuda") < 0.66, -math.inf)
        scores = -20 * torch.rand((r, b), generator=g, device="cuda").sort(1)[0]
        done = torch.zeros((r, b), dtype=torch.bool)
        for i in range(r):
            done[i, torch.from_numpy(rng.permutation(b)[:case["finished"]])] = True
        st.update(logits=logits, scores=scores, done=done.cuda(), eos=2)
    return st


# ------------------------------------------------------------- the plain forms

def _frequencies(case):
    """Radians a position, in 64 bits, and the factor on cosine and sine."""
    rot, sc = case["rot_dim"], SCALING[case["scaling"]]
    kind, factor = sc["scaling"], sc.get("factor", 1.0)
    theta = THETA * factor ** (rot / (rot - 2)) if kind == "base" else THETA
    f = theta ** (-torch.arange(0, rot, 2, dtype=torch.float64, device="cuda") / rot)
    if kind == "linear":
        f = f / factor
    if kind == "bands":
        turns = sc["original"] * f / (2 * math.pi)
        keep = ((turns - sc["slow"]) / (sc["fast"] - sc["slow"])).clamp(0, 1)
        f = f * keep + f / factor * (1 - keep)
    return f, sc.get("amplitude", 1.0)


def _rotate(x, pos, case, inverse=False):
    """x [rows, heads, head_dim]: each pair turned by position times frequency."""
    f, amp = _frequencies(case)
    angle = pos.double()[:, None] * f
    angle = -angle if inverse else angle
    cos, sin = (amp * angle.cos()).float()[:, None], (amp * angle.sin()).float()[:, None]
    rot = case["rot_dim"]
    y = x.float()
    if case["interleaved"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
        turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(x.dtype)


def _plain_rope(st):
    case = st["case"]
    return tuple(_rotate(st[n], st["pos"], case, case["inverse"]) for n in ("q", "k"))


def _plain_append(st):
    case, pos = st["case"], st["pos"].long()
    page = st["table"][st["seq"].long(), pos // case["page"]].long()
    st["k_pages"][page, :, pos % case["page"]] = _rotate(st["k"], st["pos"], case)
    st["v_pages"][page, :, pos % case["page"]] = st["v"]
    return _rotate(st["q"], st["pos"], case), st["k_pages"], st["v_pages"]


def _plain_attention(st):
    case, n = st["case"], max(1, st["longest"])
    kv, hd, ps = case["kv_heads"], case["head_dim"], case["page"]
    rows, heads = st["q"].shape[:2]
    key = torch.arange(n, device="cuda")
    page = st["table"][:, key // ps].long()
    seen = (key < st["lens"][:, None]) & (page >= 0)
    if case["window"]:
        seen &= key >= st["lens"][:, None] - case["window"]
    page = page.clamp(min=0)
    k = st["k_pages"][page, :, key % ps].float().transpose(1, 2)       # rows, kv heads, keys, head_dim
    q = st["q"].float().reshape(rows, kv, heads // kv, hd) / math.sqrt(hd)
    s = torch.matmul(q, k.transpose(2, 3))
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = (s - top.clamp(min=-1e30)).exp()
    total = p.sum(-1, keepdim=True)
    del k, s
    v = st["v_pages"][page, :, key % ps].float().transpose(1, 2)
    v = v.masked_fill(~seen[:, None, :, None], 0.0)
    out = torch.matmul(p, v) / total.clamp(min=1e-30)
    lse = (top + total.log()).reshape(rows, heads)
    return out.reshape(rows, heads, hd).to(st["q"].dtype), lse


def _plain_fork(table, ref, lens, parent):
    rows = table.shape[0]
    ok = (parent >= 0) & (parent < rows)
    at = parent.clamp(0, rows - 1).long()
    children = torch.zeros(rows, dtype=torch.int64, device="cuda").index_add_(0, at, ok.long())
    held = table >= 0
    more = torch.zeros_like(ref).index_add_(0, table.clamp(min=0).long().flatten(),
                                            ((children[:, None] - 1) * held).flatten().int())
    return torch.where(ok[:, None], table[at], -1), ref + more, torch.where(ok, lens[at], 0)


def _plain_reserve(table, ref, lens, n_new, ps):
    rows, width = table.shape
    first, end = lens // ps, (lens + n_new + ps - 1) // ps
    have = (lens + ps - 1) // ps
    page = table.gather(1, first.clamp(max=width - 1).long()[:, None])[:, 0]
    part = (lens % ps != 0) & (n_new > 0)
    same = (page[:, None] == page[None]) & part[:, None] & part[None]
    rank = same.tril(-1).sum(1)                 # writers of the same page before this one
    copy = part & ((page < 0) | (rank < ref[page.clamp(min=0).long()] - 1))
    need = copy.long() + torch.where(n_new > 0, end - have, 0)
    start = need.cumsum(0) - need
    free = (ref == 0).nonzero()[:, 0]
    short = (need.sum() - len(free)).clamp(min=0)
    go = (short == 0) & (end <= width).all()
    # page j of a sequence's new ones
    j = torch.arange(width, device="cuda") - have[:, None]
    is_new = (j >= 0) & (j < (end - have)[:, None]) & (n_new > 0)[:, None]
    is_copy = copy[:, None] & (torch.arange(width, device="cuda") == first[:, None])
    nth = torch.where(is_copy, 0, j + copy.long()[:, None]) + start[:, None]
    taken = (is_new | is_copy) & go
    got = free[nth.clamp(0, len(free) - 1)].int()
    dst = torch.where(copy, free[start.clamp(max=len(free) - 1)], -1).int()
    table2 = torch.where(taken, got, table)
    one = torch.ones_like(ref)
    ref2 = ref.index_add(0, got[taken].long(), one[:1].expand(int(taken.sum())))
    moved = copy & (page >= 0) & go
    ref2 = ref2.index_add(0, page[moved].long(), -one[:1].expand(int(moved.sum())))
    order = (~moved).long().argsort(stable=True)
    count = moved.sum()
    in_list = torch.arange(rows, device="cuda") < count
    src = torch.where(in_list, page[order], -1)
    to = torch.where(in_list, dst[order], -1)
    tokens = torch.where(in_list, (lens % ps)[order], 0)
    granted = go & (n_new > 0)
    state = torch.stack((count, need.sum() * go, short, count * 0)).int()
    return table2, ref2, lens + n_new * go, torch.where(granted, lens, -1), src, to, tokens, state


def _plain_copy(pool, src, dst, tokens):
    src, dst = src[src >= 0].long(), dst[src >= 0].long()
    if tokens is None:
        pool[:, dst] = pool[:, src]
    else:
        slot = torch.arange(pool.shape[3], device="cuda")
        keep = (slot < tokens[:len(src), None])[None, :, None, :, None]
        pool[:, dst] = torch.where(keep, pool[:, src], pool[:, dst])


def _plain_step(st):
    table, ref, lens = _plain_fork(st["table"], st["ref"], st["lens"], st["parent"])
    table, ref, lens, pos, src, dst, tokens, state = _plain_reserve(table, ref, lens, st["n_new"], st["page"])
    _plain_copy(st["k_pool"], src, dst, tokens)
    _plain_copy(st["v_pool"], src, dst, tokens)
    return table, ref, lens, pos, src, dst, tokens, state, st["k_pool"], st["v_pool"]


def _plain_compact(st):
    table, ref = st["table"], st["ref"]
    n = len(ref)
    live = ref > 0
    count = live.sum()
    page = torch.arange(n, device="cuda")
    mover, hole = live & (page >= count), ~live & (page < count)
    src, dst = mover.nonzero()[:, 0], hole.nonzero()[:, 0]
    new = torch.where(live, page, -1)
    new[src] = dst
    new = new.int()
    ref2 = ref.clone()
    ref2[dst] = ref[src]
    ref2[src] = 0
    table2 = torch.where(table >= 0, new[table.clamp(min=0).long()], -1)
    fill = torch.full((n // 2,), -1, dtype=torch.int32, device="cuda")
    a, b = fill.clone(), fill.clone()
    a[:len(src)], b[:len(src)] = src.int(), dst.int()
    _plain_copy(st["k_pool"], a, b, None)
    _plain_copy(st["v_pool"], a, b, None)
    state = torch.stack((mover.sum(), count, count * 0, count * 0)).int()
    return table2, ref2, new, a, b, state, st["k_pool"], st["v_pool"]


def _plain_beam(st):
    requests, beams = st["scores"].shape
    x = st["logits"].double()                   # in 64 bits: a candidate next to another decides whole numbers
    vocab = x.shape[1]
    top = x.amax(1, keepdim=True)
    logp = x - top - (x - top).exp().sum(1, keepdim=True).log()
    total = st["scores"].double().reshape(-1, 1) + logp
    stay = torch.full_like(total, -math.inf)
    stay[:, st["eos"]] = st["scores"].double().flatten()
    total = torch.where(st["done"].reshape(-1, 1), stay, total)
    total = torch.where(total.isnan(), -math.inf, total).reshape(requests, beams * vocab)
    best, at = total.sort(dim=1, descending=True, stable=True)
    best, at = best[:, :beams], at[:, :beams]
    beam, token = at // vocab, at % vocab
    parent = torch.arange(requests, device="cuda")[:, None] * beams + beam
    done = st["done"].gather(1, beam) | (token == st["eos"])
    return parent.int(), token.int(), best.float(), done


# ------------------------------------------------------------ one pass of a case

def _own(st):
    from paper_2606_29223_amd import paged
    kind, case = st["kind"], st["case"]
    if kind == "rope":
        return paged.rope(st["rotary"], st["pos"], st["q"], st["k"], inverse=case["inverse"])
    if kind == "append":
        q = paged.append(st["k_pages"], st["v_pages"], st["table"], st["pos"], st["k"], st["v"], seq=st["seq"],
                         rotary=st["rotary"], q=st["q"])
        return q, st["k_pages"], st["v_pages"]
    if kind == "attention":
        return paged.attention(st["q"], st["k_pages"], st["v_pages"], st["table"], st["lens"], max_len=st["longest"],
                               window=case["window"], group=case["group"], return_lse=True)
    if kind == "step":
        table, ref, lens = paged.fork(st["table"], st["ref"], st["lens"], st["parent"], out=st["next"])
        got = paged.reserve(table, ref, lens, st["n_new"], st["page"])
        paged.copy(st["k_pool"], st["v_pool"], got.src, got.dst, got.state, got.tokens)
        return table, ref, lens, got.pos, got.src, got.dst, got.tokens, got.state, st["k_pool"], st["v_pool"]
    if kind == "compact":
        table, ref = st["next"]
        got = paged.compact(st["table"], st["ref"], out=st["next"])
        paged.copy(st["k_pool"], st["v_pool"], got.src, got.dst, got.state)
        return table, ref, got.new, got.src, got.dst, got.state, st["k_pool"], st["v_pool"]
    return paged.beam_select(st["logits"], st["scores"], done=st["done"], eos=st["eos"])


PLAIN = {"rope": _plain_rope, "append": _plain_append, "attention": _plain_attention, "step": _plain_step,
         "compact": _plain_compact, "beam": _plain_beam}


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["kind"]](state)


# ---------------------------------------------------- the definitions in 64 bits

def _turned(x, pos, case, inverse=False):
    """A rotation as a complex product, row by row of frequencies."""
    rot, sc = case["rot_dim"], SCALING[case["scaling"]]
    f = []
    for i in range(rot // 2):
        base = THETA * sc["factor"] ** (rot / (rot - 2.0)) if sc["scaling"] == "base" else THETA
        v = math.exp(-2.0 * i / rot * math.log(base))
        if sc["scaling"] == "linear":
            v /= sc["factor"]
        if sc["scaling"] == "bands":
            n = sc["original"] * v / math.tau
            w = min(1.0, max(0.0, (n - sc["slow"]) / (sc["fast"] - sc["slow"])))
            v = w * v + (1.0 - w) * v / sc["factor"]
        f.append(v)
    f = torch.tensor(f, dtype=torch.float64, device="cuda")
    t = torch.polar(torch.full((len(pos), rot // 2), sc.get("amplitude", 1.0), dtype=torch.float64, device="cuda"),
                    (-1.0 if inverse else 1.0) * pos.double()[:, None] * f)[:, None]
    y = x.double().clone()
    if case["interleaved"]:
        z = torch.view_as_complex(y[..., :rot].reshape(*y.shape[:-1], rot // 2, 2).contiguous()) * t
        y[..., :rot] = torch.view_as_real(z).reshape(*y.shape[:-1], rot)
    else:
        z = torch.complex(y[..., :rot // 2], y[..., rot // 2:rot]) * t
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    return y


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "rope":
        return tuple(_turned(st[n], st["pos"], case, case["inverse"]) for n in ("q", "k"))
    if kind == "append":
        k, v = st["k_pages"].double(), st["v_pages"].double()
        page = st["table"].cpu()[st["seq"].cpu().long(), st["pos"].cpu().long() // case["page"]].long().cuda()
        slot = (st["pos"] % case["page"]).long()
        for h in range(case["kv_heads"]):
            k[page, h, slot] = _turned(st["k"][:, h:h + 1], st["pos"], case)[:, 0]
            v[page, h, slot] = st["v"][:, h].double()
        return _turned(st["q"], st["pos"], case), k, v
    if kind == "attention":
        rows, heads, hd = st["q"].shape
        kv, ps = case["kv_heads"], case["page"]
        out = torch.zeros((rows, heads, hd), dtype=torch.float64, device="cuda")
        lse = torch.full((rows, heads), -math.inf, dtype=torch.float64, device="cuda")
        for r, n in enumerate(st["lens"].tolist()):
            if n == 0:
                continue
            first = max(0, n - case["window"]) if case["window"] else 0
            pages = st["table"][r, :-(-n // ps)].long()
            k = st["k_pages"][pages].double().transpose(0, 1).reshape(kv, -1, hd)[:, first:n]
            v = st["v_pages"][pages].double().transpose(0, 1).reshape(kv, -1, hd)[:, first:n]
            for h in range(heads):
                s = (k[h * kv // heads] @ st["q"][r, h].double()) * hd ** -0.5
                lse[r, h] = torch.logsumexp(s, 0)
                out[r, h] = torch.softmax(s, 0) @ v[h * kv // heads]
        return out, lse
    if kind == "beam":
        x = st["logits"].double()
        logp = torch.log_softmax(x, 1).reshape(*st["scores"].shape, -1)
        best = []
        for r in range(case["requests"]):       # the live beams' continuations, and the finished ones as they are
            s, d = st["scores"][r].double(), st["done"][r]
            all_of = torch.cat(((s[:, None] + logp[r])[~d].flatten(), s[d]))
            best.append(all_of.topk(case["beams"])[0])
        return None, None, torch.stack(best), None
    # step and compact move values and compute none
    return None
