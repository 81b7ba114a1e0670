"""GPU: a step of drafted trees where reserve grants a sequence nothing, because it
asks for nothing or because the pages ran out: it stays as it is to the last
bit, its pages those that others share too, and the others go on."""
import numpy as np
import pytest

from tests.gpu_common import torch_cuda
from tests.paged_common import host, ints
from tests.test_gpu_trees_loop import H, HD, KV, PS, S, T, Model, Trees, guesses

pytestmark = pytest.mark.gpu


class Granted(Trees):
    """The documented step: places, lengths and paths of what was granted."""

    def __init__(self, model, start, n_pages=64):
        super().__init__(model, start, n_pages)
        self.token = ints(start)

    def step(self):
        torch, paged, c = self.torch, self.paged, self.cache
        self.drafted[:, 0] = self.token
        mask, depth = paged.tree_mask(self.parent)
        before = c.lens.clone()
        place = c.reserve(self.n_new).places(T).flatten()
        granted = c.lens - before
        at = (before[:, None] + depth).flatten()
        h = self.model.emb[self.drafted.flatten().long()]
        for l, (wi, wo) in enumerate(self.model.w):
            x = (h @ wi).view(S * T, H + 2 * KV, HD)
            q, k = paged.rope(self.plan, at, x[:, :H], x[:, H:H + KV])
            q = c.append(l, place, q, k, x[:, H + KV:], seq=self.seq)
            h = h + c.tree_attention(l, q, before, mask, n_draft=granted).flatten(1) @ wo
        target = (h @ self.model.head).argmax(1).int().view(S, T)
        path, count, token = paged.tree_accept(self.parent, self.drafted, target, n_draft=granted, root=self.token)
        c.accept(before, path, count)
        self.path.copy_(path)
        self.count.copy_(count)
        self.token.copy_(token)

    def held(self, s):
        """A sequence's keys and values, its pages, length and next token."""
        c, n = self.cache, int(self.cache.lens[s])
        pages = host(c.table)[s, :-(-n // PS)]
        rows = [np.moveaxis(host(x)[:, pages], 3, 2).reshape(x.shape[0], -1, KV, HD)[:, :n] for x in (c.k, c.v)]
        return rows + [host(c.table)[s].copy(), n, int(self.token[s])]


def same(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b))


def counted(cache):
    table = host(cache.table)
    return np.array_equal(np.bincount(table[table >= 0], minlength=len(cache.ref)), host(cache.ref))


def test_places():
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    table, ref, lens = ints(np.full((4, 6), -1)), ints(np.zeros(9)), ints([0, 3, 8, 1])
    table[1, 0], table[2, :2], table[3, 0] = 0, ints([1, 2]), 3
    ref[:4] = 1
    got = paged.reserve(table, ref, lens, ints([3, 0, 5, 2]), 4)
    place = got.places(5)
    assert place.dtype is torch.int32 and place.is_contiguous()
    assert host(place).tolist() == [[0, 1, 2, 3, 4], [-1] * 5, [8, 9, 10, 11, 12], [1, 2, 3, 4, 5]]
    got = paged.reserve(table, ref, lens, ints([20, 1, 1, 1]), 4)           # more than there are
    assert int(got.state[2]) > 0 and (host(got.places(3)) == -1).all()


@pytest.mark.parametrize("captured", [False, True])
def test_an_idle_sequence_among_trees(captured):
    """Each sequence in turn asks for nothing; the tokens of all are those that
    single steps give."""
    torch = torch_cuda()
    model, start, n = Model(4), [5, 9, 40], 30
    known = [model.greedy(t, n) for t in start]
    loop, rng = Granted(model, start), np.random.default_rng(7)
    done, got = [0] * S, [[t] for t in start]
    graph = None
    for i in range(12):
        loop.guess(*guesses(rng, known, done))
        tokens = host(loop.drafted).copy()
        idle = i % (S + 1)                                   # S: none
        loop.n_new.copy_(ints([0 if s == idle else T for s in range(S)]))
        before = [loop.held(s) for s in range(S)]
        if captured and i == 4:
            state = (loop.token, loop.cache.k, loop.cache.v, loop.cache.table, loop.cache.ref, loop.cache.lens)
            kept = [t.clone() for t in state]
            loop.step()                                      # (warm)
            graph = torch.cuda.CUDAGraph()
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                loop.step()
            for t, k in zip(state, kept):
                t.copy_(k)
        if graph is None:
            loop.step()
        else:
            graph.replay()
        path, count, after = host(loop.path), host(loop.count), host(loop.token)
        for s in range(S):
            if s == idle:
                assert count[s] == 0 and (path[s] == -1).all() and same(before[s], loop.held(s))
            else:
                assert count[s] >= 1
                got[s] += [int(tokens[s, j]) for j in path[s, 1:count[s]]] + [int(after[s])]
                done[s] += int(count[s])
        assert np.array_equal(host(loop.cache.lens), done) and counted(loop.cache)
    for s in range(S):
        m = min(len(got[s]), n + 1)
        assert m > 5 and got[s][:m] == known[s][:m]


def test_trees_when_the_pages_run_out():
    """Sequences that share their first pages, and a pool too small for their
    trees: nothing changes until there are pages again."""
    torch_cuda()
    model, start = Model(5), [5, 9, 40]
    known = [model.greedy(t, 30) for t in start]
    loop, rng = Granted(model, start, n_pages=13), np.random.default_rng(8)
    loop.n_new.copy_(ints([T, 0, 0]))
    done = [0] * S
    while done[0] < 9:                                       # one sequence alone, two shared pages and more
        loop.guess(*guesses(rng, known, done))
        loop.step()
        done[0] = int(loop.cache.lens[0])
    loop.cache.fork(ints([0, 0, -1]))
    loop.token[1] = loop.token[0]
    before = [loop.held(s) for s in range(S)]
    pool = [host(loop.cache.k), host(loop.cache.v)]
    ref = host(loop.cache.ref).copy()
    loop.cache.ref[loop.cache.ref == 0] = 1                  # someone else has the free pages
    loop.n_new.fill_(T)
    for _ in range(2):
        loop.guess(*guesses(rng, known, done))
        loop.step()
        assert (host(loop.count) == 0).all() and all(same(a, loop.held(s)) for s, a in enumerate(before))
        assert np.array_equal(pool[0], host(loop.cache.k)) and np.array_equal(pool[1], host(loop.cache.v))
    loop.cache.ref.copy_(ints(ref))
    loop.step()
    assert (host(loop.count) >= 1).all() and counted(loop.cache)
    n = int(before[0][3])
    for s in (0, 1):
        now = loop.held(s)
        assert now[3] > n and np.array_equal(now[0][:, :n], before[0][0]) and np.array_equal(now[1][:, :n], before[0][1])


def test_accept_leaves_what_was_not_granted():
    """Paths of whole trees, asked for without the numbers granted: a sequence
    that was granted nothing keeps its tokens and its length."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    cache = paged.PagedCache(2, KV, HD, PS, 20, 3, 8, dtype=torch.float32)
    cache.reserve(ints([6, 9, 3]))
    cache.k.copy_(torch.randn_like(cache.k))
    cache.v.copy_(torch.randn_like(cache.v))
    k, table, before = host(cache.k), host(cache.table), cache.lens.clone()
    cache.reserve(ints([5, 0, 5]))
    path = ints([[0, 2, 4, -1, -1], [0, 3, -1, -1, -1], [1, -1, -1, -1, -1]])
    cache.accept(before, path, ints([3, 2, 1]))
    assert host(cache.lens).tolist() == [9, 9, 4] and np.array_equal(host(cache.table)[1], table[1])
    assert np.array_equal(host(cache.k)[:, table[1, :3]], k[:, table[1, :3]]) and counted(cache)
