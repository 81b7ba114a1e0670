"""GPU: rows that attend in groups and end at a split's edge.  A row of 256 keys
is one split, a longer row that begins with the same pages has several; whoever
reads the shared split, each row gets it where its own join looks for it.
Outputs are full of NaN before the call, and so is the memory that it works in."""
import itertools

import numpy as np
import pytest

from oracle import paged as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import attention_bounds, host, ints, normal

pytestmark = pytest.mark.gpu

PAGE, KV = 16, 2
GROUPS = [(256, 300), (300, 256), (255, 256, 257), (257, 256, 255), (256, 256, 257), (6144, 256), (256, 6144),
          (512, 513, 512), (513, 256, 512), (64 * 95, 64 * 96, 64 * 97), (64 * 97, 256, 64 * 96), (256, 0, 300),
          (0, 256, 300), (300, 256, 256, 1000)]


def _nan_memory(torch):
    """The allocator's next blocks hold NaN (work memory comes from them)."""
    blocks = [torch.full((n,), float("nan"), device="cuda") for n in (1 << 10, 1 << 16, 1 << 18, 1 << 20, 1 << 22, 1 << 24)]
    torch.cuda.synchronize()
    del blocks


class Shared:
    """Rows of one group whose keys are the same as far as they go: by pages of
    their own table rows, or as rows of one sequence."""

    def __init__(self, seed, dtype, hd, H, lens, one_sequence):
        self.rng, self.dtype, self.hd = np.random.default_rng(seed), dtype, hd
        self.lens = np.array(lens)
        n = -(-max(lens) // PAGE)
        ids = self.rng.permutation(n + 3)[:n]
        if one_sequence:
            self.table, self.seq = ids[None], np.zeros(len(lens), int)
        else:
            self.table, self.seq = np.full((len(lens), n), -1), None
            for r, v in enumerate(lens):
                self.table[r, :-(-v // PAGE)] = ids[:-(-v // PAGE)]
        self.k, self.k64 = normal(self.rng, (n + 3, KV, PAGE, hd), dtype)
        self.v, self.v64 = normal(self.rng, (n + 3, KV, PAGE, hd), dtype)
        self.q, self.q64 = normal(self.rng, (len(lens), H, hd), dtype, 1.5)

    def run(self, group, window=0):
        torch = torch_cuda()
        from paper_2606_29223_amd import paged
        _nan_memory(torch)
        out = torch.full_like(self.q, float("nan"))
        return paged.attention(self.q, self.k, self.v, ints(self.table), ints(self.lens), group=group, window=window, out=out,
                               seq=None if self.seq is None else ints(self.seq), return_lse=True)

    def check(self, got, window=0):
        out, lse, spread, size = ref.attention(self.q64, self.k64, self.v64, self.table, self.lens, seq=self.seq, window=window)
        tol, ltol = attention_bounds(self.q64, spread, size, out, lse, self.hd, self.dtype)
        g, l = host(got[0]), host(got[1])
        assert np.array_equal(np.isneginf(l), np.isneginf(lse))
        assert (np.abs(g - out) <= tol).all()
        ok = np.isfinite(lse)
        assert (np.abs(l[ok] - lse[ok]) <= ltol[ok]).all()


@pytest.mark.parametrize("one_sequence", [False, True])
@pytest.mark.parametrize("dtype,hd,H", [("bf16", 128, 8), ("f32", 64, 2), ("bf16", 32, 16)])
@pytest.mark.parametrize("lens", GROUPS, ids=lambda g: "-".join(map(str, g)))
def test_groups_that_end_at_a_split(lens, dtype, hd, H, one_sequence):
    """The bits of single rows, in windows that cut nothing too."""
    torch_cuda()
    c = Shared(sum(lens) + hd, dtype, hd, H, lens, one_sequence)
    alone = c.run(1)
    c.check(alone)
    for group, window in itertools.product((len(lens), 8), (0, max(lens), 1 << 20)):
        got = c.run(group, window)
        assert all(np.array_equal(host(a), host(b)) for a, b in zip(got, alone)), (group, window)
    narrow = c.run(1, 300)
    c.check(narrow, 300)
    assert all(np.array_equal(host(a), host(b)) for a, b in zip(c.run(len(lens), 300), narrow))
