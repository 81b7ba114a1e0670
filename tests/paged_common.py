"""Inputs and error bounds shared by the GPU tests of the paged-cache operators."""
import numpy as np

from tests.gpu_common import torch_cuda

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}        # one rounding, relative to the value


def dtype_of(name):
    torch = torch_cuda()
    return {"f32": torch.float32, "bf16": torch.bfloat16}[name]


def ints(a):
    torch = torch_cuda()
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def normal(rng, shape, dtype, scale=1.0):
    """A GPU tensor and its exact values in float64."""
    torch = torch_cuda()
    t = torch.from_numpy((scale * rng.standard_normal(shape)).astype(np.float32)).to(dtype_of(dtype))
    return t.cuda(), t.double().numpy()


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def random_table(rng, lens, page, spare=3):
    """A page table of shuffled pages for the lengths, -1 behind: (table, n_pages)."""
    n = [-(-int(v) // page) for v in lens]
    ids = rng.permutation(sum(n) + spare)
    table = np.full((len(lens), max(1, max(n))), -1)
    at = 0
    for s, c in enumerate(n):
        table[s, :c] = ids[at:at + c]
        at += c
    return table, len(ids)


def attention_bounds(q, spread, size, out, lse, hd, dtype):
    """Elementwise bounds of (out, lse) against float64.

    A score is a sum of hd products, each and each partial sum off by 2^-24 of
    at most `size` (the largest sum |q k| scale), then scaled and taken to
    powers of two: |ds| <= (hd + 4) 2^-24 size.  A probability is off by that
    on both sides of its quotient, by 2^-22 in its power, and in bf16 by the
    second part's rounding, 2^-17 at most.  Sums of up to 64 products in a
    tile, 4 waves and a row's records follow, each addition off by 2^-24 of
    the spread (sum of p |v|): at most 128 of them in a row.  The output is
    rounded once."""
    ds = (hd + 4) * 2.0 ** -24 * size
    p = 2 * ds + 2.0 ** -21 + 128 * 2.0 ** -24 + (2.0 ** -16 if dtype == "bf16" else 0.0)
    tol = p[..., None] * spread + (HALF_STEP[dtype] * 1.01) * np.abs(out) + 1e-30
    finite = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    return tol, ds + 2.0 ** -21 + 128 * 2.0 ** -24 + 2.0 ** -22 * (finite + size)
