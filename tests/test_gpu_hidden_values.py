"""GPU: values that a row does not see, or sees with a weight that is 0 in float,
leave its output alone however large they are, finite ones too."""
import numpy as np
import pytest

from tests.gpu_common import torch_cuda
from tests.paged_common import HALF_STEP, dtype_of, host, ints
from tests.test_gpu_tree_attention import Case, many_wide

pytestmark = pytest.mark.gpu

LARGE = [1e30, -1e30, 3.3895313892515355e38, -3.3895313892515355e38]      # the last two: the largest bf16


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("draft", [2, 3, 12, 20, 40, 64])
def test_large_drafted_values_that_only_some_rows_see(dtype, draft):
    """One block of columns a wave alone and over four waves, and (from 20 rows on)
    the same with more columns: the rows that do not see the value keep every
    bit, of the others the other dimensions do."""
    torch_cuda()
    c = Case(draft, dtype, 64, 8, 2, 16, [40, 61, 0, 31, 300], draft)
    c.seen[:] = np.eye(draft, dtype=bool)
    c.seen[:, draft // 2:, 0] = True
    clean = [host(t) for t in c.run()]
    sees = c.seen[:, :, 0].reshape(-1)
    for big in LARGE:
        for b, n in enumerate(c.lens):
            c.v[int(c.table[b, n // 16]), :, n % 16, 5] = big
        out = c.run()
        got = [host(t) for t in out]
        assert np.array_equal(got[0][~sees], clean[0][~sees]), big
        assert np.array_equal(np.delete(got[0], 5, 2), np.delete(clean[0], 5, 2)) and np.array_equal(got[1], clean[1]), big
        assert (np.sign(got[0][sees][..., 5]) == np.sign(big)).all(), big
        if abs(big) < 1e38:                                   # (no sum of weights near 2^8 overflows)
            c.v64 = host(c.v)
            c.check(out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hd,page", [(32, 4), (64, 16), (128, 2)])
def test_large_drafted_values_in_many_wide_trees(dtype, hd, page):
    """Two blocks of columns a wave, ragged trees."""
    torch_cuda()
    c = many_wide(dtype, hd, page)
    c.seen[:] = np.eye(20, dtype=bool)
    c.seen[:, 10:, 1] = True
    clean = [host(t) for t in c.run()]
    for big in LARGE:
        sees = np.zeros((20, 20), bool)
        for b, n in enumerate(c.lens):
            if c.drafts[b] > 1:
                c.v[int(c.table[b, (n + 1) // page]), :, (n + 1) % page, 7] = big
                sees[b] = c.seen[b, :, 1] & (np.arange(20) < c.drafts[b])
        got = [host(t) for t in c.run()]
        sees = sees.reshape(-1)
        assert np.array_equal(got[0][~sees], clean[0][~sees]), big
        assert np.array_equal(np.delete(got[0], 7, 2), np.delete(clean[0], 7, 2)) and np.array_equal(got[1], clean[1]), big


def _underflow(dtype, keys, at, score, value, hd=64):
    """One row over `keys` keys of score 0 and value 1, but for the one at `at`."""
    torch = torch_cuda()
    n = -(-(keys + 1) // 16)
    k, v = np.zeros((n, 1, 16, hd)), np.ones((n, 1, 16, hd))
    k[at // 16, 0, at % 16, 0] = score
    v[at // 16, 0, at % 16, 3] = value
    q = np.zeros((1, 4, hd))
    q[..., 0] = 1.0
    t = lambda a: torch.from_numpy(a).to(dtype_of(dtype)).cuda()
    return t(q), t(k), t(v), ints(np.arange(n)[None])


def _every_form(q, k, v, table, keys):
    """The same row as a tree of one token and none, chosen pages, and weights."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    mask = torch.zeros((1, 1, 1), dtype=torch.int64, device="cuda")
    columns = torch.arange(table.shape[1], dtype=torch.int32, device="cuda").expand(1, 1, -1).contiguous()
    weight = torch.zeros((1, 1, table.shape[1] * 16), device="cuda")
    yield host(paged.tree_attention(q, k, v, table, ints([keys]), mask, scale=1.0))
    yield host(paged.sparse_attention(q, k, v, table, ints([keys]), columns, scale=1.0))
    yield host(paged.weigh(q, k, v, table, ints([keys]), weight, scale=1.0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("keys,at", [(40, 3), (40, 39), (900, 500), (900, 899), (3000, 7)])
def test_large_values_whose_weight_is_zero_in_float(dtype, keys, at):
    """A key 1000 below the others: its weight is e^-1000.  Every other value is 1
    and so is the output, but for `keys` additions of 2^-24 each on both sides of
    the quotient and one rounding; in bf16 two parts of 2^-133 may stand for the
    weight, of the `keys` that the sum of weights comes to."""
    torch_cuda()
    for big in LARGE:
        for got in _every_form(*_underflow(dtype, keys, at, -1000.0, big), keys):
            tol = (2 * (keys + 128) + 8) * 2.0 ** -24 + HALF_STEP[dtype]
            if dtype == "bf16":
                tol += 2.0 ** -132 * abs(big) / keys
            assert np.abs(got - 1.0).max() <= tol, (big, np.abs(got - 1.0).max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("score", [-8.0, -40.0, -72.0, -84.0])
def test_small_weights_of_large_and_infinite_values(dtype, score):
    """Weights down to e^-84, 2^-121: a finite value counts with its weight, an
    infinite one is infinite in the output.  The score is exact; the weight is
    off by 2^-22 and by its logarithm's rounding, 2^-24 of up to 122; where that
    is near 2^-126 the parts' least step, 2^-133, is added twice at most."""
    torch_cuda()
    keys, at = 300, 100
    value = float(torch_cuda().tensor(2.0 * np.exp(-score)).bfloat16())
    p = np.exp(score)
    want = (keys - 1 + p * value) / (keys - 1 + p)
    rel = 2.0 ** -22 + 123 * 2.0 ** -24 + 2.0 ** -132 / p + 2 * (keys + 128) * 2.0 ** -24
    for got in _every_form(*_underflow(dtype, keys, at, score, value), keys):
        assert np.abs(got[..., 3] - want).max() <= rel * want + HALF_STEP[dtype] * 1.01 * want
    for bad in (float("inf"), float("-inf")):
        for got in _every_form(*_underflow(dtype, keys, at, score, bad), keys):
            assert (got[..., 3] == bad).all() and np.isfinite(np.delete(got, 3, 2)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 4])
def test_large_values_of_single_rows(dtype, group):
    """The same for attention of one token a row, alone and in a group whose
    pages are read once: weights of 0 in float, and small ones of large and
    infinite values."""
    torch_cuda()
    from paper_2606_29223_amd import paged
    keys, at = 900, 500
    run = lambda q, k, v, table: host(paged.attention(q.expand(4, -1, -1).contiguous(), k, v, table.expand(4, -1).contiguous(),
                                                      ints([keys] * 4), scale=1.0, group=group))
    for big in LARGE:
        tol = (2 * (keys + 128) + 8) * 2.0 ** -24 + HALF_STEP[dtype] + (2.0 ** -132 * abs(big) / keys if dtype == "bf16" else 0)
        assert np.abs(run(*_underflow(dtype, keys, at, -1000.0, big)) - 1.0).max() <= tol, big
    for score in (-40.0, -84.0):
        value, p = float(torch_cuda().tensor(2.0 * np.exp(-score)).bfloat16()), np.exp(score)
        want = (keys - 1 + p * value) / (keys - 1 + p)
        rel = 2.0 ** -22 + 123 * 2.0 ** -24 + 2.0 ** -132 / p + 2 * (keys + 128) * 2.0 ** -24
        got = run(*_underflow(dtype, keys, at, score, value))
        assert np.abs(got[..., 3] - want).max() <= rel * want + HALF_STEP[dtype] * 1.01 * want
        for bad in (float("inf"), float("-inf")):
            got = run(*_underflow(dtype, keys, at, score, bad))
            assert (got[..., 3] == bad).all() and np.isfinite(np.delete(got, 3, 2)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("score", [0.0, 32.0, -32.0])
def test_infinite_values_with_weights_of_few_bits(dtype, score):
    """The row's largest key has weight 1, whose lower parts are nothing, and one
    value of it is infinite."""
    torch_cuda()
    for keys, at in ((40, 3), (900, 500), (900, 899)):
        for bad in (float("inf"), float("-inf")):
            for got in _every_form(*_underflow(dtype, keys, at, score, bad), keys):
                assert (got[..., 3] == bad).all() and np.isfinite(np.delete(got, 3, 2)).all()
