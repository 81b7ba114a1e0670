"""GPU: the paged-cache operators together, as a decoding loop with beams uses
them: reserve, rotate and write, attend, select, fork -- against the float64
references step by step, captured into a graph and replayed, on another stream
and with the pages compacted on the way."""
import numpy as np
import pytest

from oracle import paged as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import host, ints

pytestmark = pytest.mark.gpu

R, B, H, KV, HD, L, PS, V = 2, 3, 4, 2, 32, 2, 4, 301


class Loop:
    """A toy model around the operators: token -> embedding -> per layer
    (projections, append, attention, residual) -> logits."""

    def __init__(self, seed=1, n_pages=64):
        torch = torch_cuda()
        from paper_2606_29223_amd import paged
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.torch, self.paged = torch, paged
        rnd = lambda *s: torch.randn(s, generator=g, device="cuda") / s[0] ** 0.5
        self.emb = rnd(V, H * HD) * V ** 0.5
        self.w = [(rnd(H * HD, (H + 2 * KV) * HD), rnd(H * HD, H * HD)) for _ in range(L)]
        self.head = rnd(H * HD, V) * 3
        self.plan = paged.Rotary(HD, interleaved=True)
        self.cache = paged.PagedCache(L, KV, HD, PS, n_pages, R * B, 16, dtype=torch.float32)
        self.score = torch.tensor([[0.0] + [-np.inf] * (B - 1)] * R, device="cuda")
        self.done = torch.zeros((R, B), dtype=torch.bool, device="cuda")
        self.token = torch.tensor([[5] * B, [9] * B], dtype=torch.int32, device="cuda")
        self.one = torch.ones(R * B, dtype=torch.int32, device="cuda")
        self.parent = torch.empty((R, B), dtype=torch.int32, device="cuda")

    def step(self):
        c, paged = self.cache, self.paged
        pos = c.reserve(self.one).pos
        h = self.emb[self.token.flatten().long()]
        for l, (wi, wo) in enumerate(self.w):
            x = (h @ wi).view(R * B, H + 2 * KV, HD)
            q = c.append(l, pos, x[:, :H], x[:, H:H + KV], x[:, H + KV:], rotary=self.plan)
            h = h + c.attention(l, q, group=B).flatten(1) @ wo
        logits = h @ self.head
        parent, token, score, done = paged.beam_select(logits, self.score, done=self.done, eos=3)
        c.fork(parent.flatten())
        self.token.copy_(token)
        self.score.copy_(score)
        self.done.copy_(done)
        self.parent.copy_(parent)
        return logits

    def state(self):
        c = self.cache
        return [host(t).copy() for t in (self.token, self.score, self.done, self.parent, c.table, c.ref, c.lens)]


def _plain(loop, steps):
    """The same loop with every beam's whole history attended to afresh in
    float64: tokens, parents and scores of each step."""
    emb, head = host(loop.emb), host(loop.head)
    w = [(host(a), host(b)) for a, b in loop.w]
    freq = ref.frequencies(HD)
    hist = [[5], [5], [5], [9], [9], [9]]
    score = np.array([[0.0, -np.inf, -np.inf]] * R)
    done = np.zeros((R, B), bool)
    out = []
    for _ in range(steps):
        logits = np.zeros((R * B, V))
        for r, toks in enumerate(hist):
            n = len(toks)
            h = emb[toks]
            for wi, wo in w:
                x = (h @ wi).reshape(n, H + 2 * KV, HD)
                q = ref.rotate(x[:, :H], np.arange(n), freq, True)
                k = ref.rotate(x[:, H:H + KV], np.arange(n), freq, True)
                o = np.zeros((n, H, HD))
                for i in range(n):
                    for a in range(H):
                        s = k[:i + 1, a // 2] @ q[i, a] / HD ** 0.5
                        p = np.exp(s - s.max())
                        o[i, a] = p @ x[:i + 1, H + KV + a // 2] / p.sum()
                h = h + o.reshape(n, -1) @ wo
            logits[r] = h[-1] @ head
        parent, token, score, ends = ref.beam_select(logits, score.astype(np.float32), B, done, 3)
        done = ends
        hist = [hist[p] + [int(t)] for p, t in zip(parent.flatten(), token.flatten())]
        out.append((parent, token, score, logits))
    return out


def test_beam_decoding_against_whole_histories():
    loop = Loop()
    want = _plain(loop, 14)
    for i, (parent, token, score, logits) in enumerate(want):
        got = loop.step()
        live = np.isfinite(score)
        assert np.array_equal(host(loop.parent), parent) and np.array_equal(host(loop.token), token), i
        # float matrix products of 128 terms, two layers deep, summed over the steps
        assert np.abs(host(loop.score) - score)[live].max() < 1e-3
        if i % 5 == 4:
            before = host(loop.cache.ref)
            loop.cache.compact()
            assert sorted(before) == sorted(host(loop.cache.ref))
    counts = np.bincount(host(loop.cache.table)[host(loop.cache.table) >= 0], minlength=64)
    assert np.array_equal(counts, host(loop.cache.ref))
    loop.cache.fork(ints([-1] * (R * B)))                 # everything is freed
    assert (host(loop.cache.ref) == 0).all() and (host(loop.cache.lens) == 0).all()


def test_a_captured_step_replays():
    """One captured step, replayed with eager work in between, goes through the
    same states as the eager loop, bit for bit."""
    torch = torch_cuda()
    eager, loop = Loop(), Loop()
    for _ in range(2):
        eager.step()
        loop.step()
    assert all(np.array_equal(a, b, equal_nan=True) for a, b in zip(eager.state(), loop.state()))
    before = [t.clone() for t in (loop.token, loop.score, loop.done, loop.cache.k, loop.cache.v, loop.cache.table,
                                  loop.cache.ref, loop.cache.lens)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        loop.step()                                       # the products' workspaces exist before the capture
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loop.step()
    for t, b in zip((loop.token, loop.score, loop.done, loop.cache.k, loop.cache.v, loop.cache.table, loop.cache.ref,
                     loop.cache.lens), before):
        t.copy_(b)
    for i in range(9):
        eager.step()
        graph.replay()
        if i % 3 == 1:
            torch.cuda.synchronize()
        assert all(np.array_equal(a, b, equal_nan=True) for a, b in zip(eager.state(), loop.state())), i
        assert torch.equal(eager.cache.k, loop.cache.k) and torch.equal(eager.cache.v, loop.cache.v)


def test_two_loops_on_two_streams():
    torch = torch_cuda()
    want = []
    for seed in (1, 2):
        loop = Loop(seed)
        for _ in range(8):
            loop.step()
        want.append(loop.state())
    loops, streams = [Loop(1), Loop(2)], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(8):
        for loop, s in zip(loops, streams):
            with torch.cuda.stream(s):
                loop.step()
    torch.cuda.synchronize()
    for loop, w in zip(loops, want):
        assert all(np.array_equal(a, b, equal_nan=True) for a, b in zip(loop.state(), w))


def test_a_full_cache_grants_nothing():
    """Out of pages: the step's rows have no place, nothing of the cache
    changes, and after a sequence is freed it goes on."""
    loop = Loop(n_pages=8)
    torch = torch_cuda()
    c = loop.cache
    grown = 0
    for _ in range(60):
        was = [host(t) for t in (c.table, c.ref, c.lens, c.k)]
        got = c.reserve(loop.one)
        if host(got.state)[2]:
            assert (host(got.pos) == -1).all()
            assert all(np.array_equal(a, host(t)) for a, t in zip(was, (c.table, c.ref, c.lens, c.k)))
            x = torch.ones((R * B, KV, HD), device="cuda")
            assert c.append(0, got.pos, None, x, x) is None
            assert np.array_equal(was[3], host(c.k))
            break
        grown += 1
    assert grown == 4                                     # eight pages: a page of four tokens each of six sequences
    c.fork(ints([0, 1, 2, -1, -1, -1]))
    got = c.reserve(ints([1, 1, 1, 0, 0, 0]))
    assert host(got.state).tolist() == [0, 3, 0, 0] and host(got.pos).tolist() == [4, 4, 4, -1, -1, -1]


def test_the_binding_refuses_numbers_and_outputs_that_do_not_fit():
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    from paper_2606_29223_amd.dexlib import DEX_E_INVAL, DexError
    cache = paged.PagedCache(1, 2, 32, 8, 6, 3, 4)
    x, pos = torch.zeros((3, 2, 32), dtype=torch.bfloat16, device="cuda"), torch.zeros_like(cache.lens)
    one = torch.zeros((1, 2, 32), dtype=torch.bfloat16, device="cuda").expand(3, 2, 32)
    plan = paged.Rotary(32)
    logits, score = torch.zeros((6, 50), device="cuda"), torch.zeros((3, 2), device="cuda")
    for call in (lambda: paged.rope(plan, pos, x, q_out=one), lambda: cache.attention(0, x, out=one),
                 lambda: cache.attention(0, x, group=2 ** 32 + 1), lambda: cache.attention(0, x, window=2 ** 32),
                 lambda: cache.attention(0, x, max_len=-(2 ** 32)), lambda: cache.append(0, pos, x[:2], x, x),
                 lambda: paged.reserve(cache.table, cache.ref, cache.lens, pos, 2 ** 32 + 8),
                 lambda: cache.fork(pos.long()), lambda: cache.fork(pos[:2]), lambda: cache.reserve(pos.cpu()),
                 lambda: paged.beam_select(logits, score, eos=2 ** 32), lambda: paged.beam_select(logits, score, eos=50),
                 lambda: paged.beam_select(logits, score, n_out=10 ** 12),
                 lambda: paged.beam_select(logits[:5], score)):
        with pytest.raises(DexError) as e:
            call()
        assert e.value.status == DEX_E_INVAL
    assert torch.equal(paged.rope(plan, pos, one), x)      # an input may be a broadcast one
