"""GPU: the weights of attention reach the values with all their bits, and an
infinite value that is attended to is one in the output."""
import numpy as np
import pytest

from tests.gpu_common import torch_cuda
from tests.paged_common import HALF_STEP, dtype_of, host, ints

pytestmark = pytest.mark.gpu

LN2 = float(np.log(2.0))


def _bf16(x):
    torch = torch_cuda()
    return torch.from_numpy(np.asarray(x, np.float32)).bfloat16().double().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd", [32, 64, 128])
def test_weights_have_all_their_bits(dtype, hd):
    """Three keys with scores 0, 0 and -x and values 1, v and -c that cancel to
    2^-18, where the output's own rounding says nothing: what is left is the
    error of p = e^-x.  Scores are exact; x log2 e < 2 is rounded once (2^-24)
    with a constant that is off by 2^-26 of it, the power is good to 2^-23, and
    five sums of terms up to 1 follow, each off by 2^-24 at most, and one more
    in l."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    x = _bf16(np.linspace(0.11, 1.37, 160))
    p = np.exp(-x)
    c = _bf16(np.linspace(0.9, 1.1, hd)[None] / p[:, None])        # another value in each dimension
    rows = len(x)
    k, v = np.zeros((rows, 1, 4, hd)), np.zeros((rows, 1, 4, hd))
    k[:, 0, 2, 0] = -x
    v[:, 0, 0], v[:, 0, 2] = 1.0, -c
    v[:, 0, 1] = _bf16(p[:, None] * c - 1.0)
    q = np.zeros((rows, 1, hd))
    q[..., 0] = 1.0
    t = lambda a: torch.from_numpy(a).to(dtype_of(dtype)).cuda()
    got = host(paged.attention(t(q), t(k), t(v), ints(np.arange(rows)[:, None]), ints(np.full(rows, 3)), scale=1.0))[:, 0]
    l = (2.0 + p)[:, None]
    want = (v[:, 0, 0] + v[:, 0, 1] + p[:, None] * v[:, 0, 2]) / l
    dp = p[:, None] * (2.0 ** -23 + LN2 * (2.0 ** -24 + 2.0 ** -25))
    tol = (dp * c + 6 * 2.0 ** -24) / l + HALF_STEP[dtype] * 1.01 * np.abs(want)
    assert (np.abs(got - want) <= tol).all(), np.max(np.abs(got - want) / tol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("H", [4, 48])
def test_infinite_values_that_are_attended_to(dtype, H):
    """Infinity where one attended value is infinite, NaN where two of unlike
    sign or a NaN are; other dimensions and sequences as if it were not there."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(3)
    lens, hd = [1, 40, 300, 1500], 64
    pages = [-(-n // 16) for n in lens]
    table, at = np.full((4, max(pages)), -1), 0
    for s, n in enumerate(pages):
        table[s, :n] = np.arange(at, at + n)
        at += n
    t = lambda a: torch.from_numpy(a.astype(np.float32)).to(dtype_of(dtype)).cuda()
    k, v, q = t(rng.standard_normal((at, 2, 16, hd))), t(rng.standard_normal((at, 2, 16, hd))), t(rng.standard_normal((4, H, hd)))
    run = lambda: host(paged.attention(q, k, v, ints(table), ints(lens)))
    want = run()
    for s, n in enumerate(lens):
        first, last = table[s, 0], table[s, (n - 1) // 16]
        v[last, :, (n - 1) % 16, 5] = float("inf")
        v[last, 0, (n - 1) % 16, 9] = float("-inf")
        v[first, :, 0, 11] = float("nan")
        want[s, :, 5] = np.inf
        want[s, :H // 2, 9] = -np.inf
        want[s, :, 11] = np.nan
        if n > 1:
            v[first, :, 0, 7], v[last, :, (n - 1) % 16, 7] = float("inf"), float("-inf")
            want[s, :, 7] = np.nan
    assert np.array_equal(run(), want, equal_nan=True)
