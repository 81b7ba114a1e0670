"""GPU: rotary positions (dex_rope) and the cache write with them
(dex_pages_append) against float64.

Bounds: cosine and sine are off by at most 2^-22 (2^-25 of the angle's float,
the series' roundings and its cut), the two products and their sum by three
more roundings of 2^-24: (|x| + |y|) amplitude 2^-21 in all, and the output by
half a step of its type.  The angle itself is pos * f with f and the product
rounded in double on both sides, 2^-50 of the position at most (f <= 1)."""
import numpy as np
import pytest

from oracle import paged as ref
from tests.gpu_common import torch_cuda
from tests.paged_common import HALF_STEP, dtype_of, host, ints, normal, random_table

pytestmark = pytest.mark.gpu


def _check(got, x, pos, freq, dtype, rot, interleaved, amplitude=1.0, inverse=False):
    want = ref.rotate(x, pos, freq, interleaved, amplitude, inverse)
    a, b = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2, rot))
    both = np.zeros(x.shape)
    both[..., a] = both[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    far = np.abs(np.asarray(pos, dtype=np.float64))[:, None, None] * 2.0 ** -50
    tol = both * amplitude * (2.0 ** -21 + far) + HALF_STEP[dtype] * 1.01 * np.abs(want)
    assert (np.abs(host(got) - want) <= tol).all(), np.max(np.abs(host(got) - want) - tol)
    assert np.array_equal(host(got)[..., rot:], x[..., rot:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,kv,hd,rot", [(1, 1, 1, 2, 2), (3, 4, 4, 32, 8), (77, 12, 12, 64, 32), (5, 3, 1, 80, 80),
                                                  (2, 7, 1, 66, 22), (300, 32, 8, 128, 128), (9, 2, 1, 256, 64)])
def test_rope_against_float64(dtype, interleaved, rows, heads, kv, hd, rot):
    torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(rows * 1000 + hd)
    q, q64 = normal(rng, (rows, heads, hd), dtype)
    k, k64 = normal(rng, (rows, kv, hd), dtype)
    pos = rng.integers(0, 1 << 20, rows)
    pos[0], pos[-1] = 0, 2 ** 31 - 1
    kw = dict(scaling="bands", factor=16.0, original=8192, slow=1, fast=32)
    plan = paged.Rotary(hd, rot_dim=rot, interleaved=interleaved, amplitude=1.277, **kw)
    freq = ref.frequencies(rot, **kw)
    for inverse in (False, True):
        a, b = paged.rope(plan, ints(pos), q, k, inverse=inverse)
        _check(a, q64, pos, freq, dtype, rot, interleaved, 1.277, inverse)
        _check(b, k64, pos, freq, dtype, rot, interleaved, 1.277, inverse)
    neg = paged.rope(plan, ints(-pos), q)                 # a negative position is a turn back
    back, _ = paged.rope(plan, ints(pos), q, k, inverse=True)
    assert np.array_equal(host(neg), host(back))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strides_alignment_and_in_place_have_the_same_bits(dtype):
    """Views of a fused projection, head-major views, odd offsets, an output in
    place or strided: the bits of dense tensors."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(5)
    rows, h, kv, hd = 13, 6, 2, 64
    pos = ints(rng.integers(0, 5000, rows))
    plan = paged.Rotary(hd)
    x, _ = normal(rng, (rows, h + 2 * kv, hd), dtype)
    q, k = x[:, :h], x[:, h:h + kv]
    want_q, want_k = paged.rope(plan, pos, q.contiguous(), k.contiguous())
    a, b = paged.rope(plan, pos, q, k)
    assert torch.equal(a, want_q) and torch.equal(b, want_k)
    flat = torch.zeros(rows * h * hd + 7, dtype=x.dtype, device="cuda")
    for off in (1, 2, 4, 7):                              # every access width
        odd = flat[off:off + rows * h * hd].view(rows, h, hd)
        odd.copy_(q)
        assert torch.equal(paged.rope(plan, pos, odd), want_q), off
        paged.rope(plan, pos, odd, q_out=odd)
        assert torch.equal(odd, want_q), off
    major = q.transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.full((rows, 2 * h, hd), 9.0, dtype=x.dtype, device="cuda")
    paged.rope(plan, pos, major, q_out=out[:, ::2])
    assert torch.equal(out[:, ::2], want_q) and (out[:, 1::2] == 9).all()
    paged.rope(plan, pos, q, k, q_out=q, k_out=k)         # in place in the fused rows
    assert torch.equal(x[:, :h], want_q) and torch.equal(x[:, h:h + kv], want_k)


def test_as_many_rows_as_a_call_takes():
    """1.3 billion rows of five fp32 heads of one pair (52 GB), close to the
    limit of a call: more lanes of four heads than an int counts."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rows = 1_300_000_000
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("less than 80 GiB of GPU memory is free")
    plan = paged.Rotary(2)
    x, _ = normal(np.random.default_rng(8), (1, 5, 2), "f32")
    pos = torch.arange(rows, dtype=torch.int32, device="cuda")
    got = paged.rope(plan, pos, x.expand(rows, 5, 2))
    some = torch.randint(0, rows, (100_000,), generator=torch.Generator().manual_seed(1)).cuda()
    some[:2] = torch.tensor([0, rows - 1])
    assert torch.equal(got[some], paged.rope(plan, pos[some], x.expand(len(some), 5, 2)))
    del got, pos
    torch.cuda.empty_cache()


def test_a_turn_back_is_the_gradient():
    """The gradient of sum(g * rope(x)) by differences, which a linear map's
    are exact to rounding: each difference of sums is off by rows * heads * hd
    roundings of 2^-24 of values up to 8."""
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(6)
    x, _ = normal(rng, (2, 1, 16), "f32")
    g, _ = normal(rng, (2, 1, 16), "f32")
    pos, plan = ints([3, 4001]), paged.Rotary(16, rot_dim=12, interleaved=True)
    grad = paged.rope(plan, pos, g, inverse=True).flatten()
    for i in range(x.numel()):
        d = torch.zeros_like(x).view(-1)
        d[i] = 0.5
        up, down = ((g.double() * paged.rope(plan, pos, x + t * d.view_as(x)).double()).sum() for t in (1, -1))
        assert abs(float(up - down) - float(grad[i])) < 64 * 8 * 2.0 ** -24


def _append_case(dtype, page, hd, rot, tokens, seed):
    torch = torch_cuda()
    from paper_2606_29223_amd import paged
    rng = np.random.default_rng(seed)
    H, kv, S = 6, 2, 4
    first = rng.integers(0, 40, S)
    table, n_pages = random_table(rng, first + tokens, page)
    kp, k64 = normal(rng, (n_pages, kv, page, hd), dtype)
    vp, v64 = normal(rng, (n_pages, kv, page, hd), dtype)
    x, x64 = normal(rng, (S * tokens, H + 2 * kv, hd), dtype)
    seq = np.repeat(np.arange(S), tokens)
    pos = (first[:, None] + np.arange(tokens)[None]).reshape(-1)
    plan = paged.Rotary(hd, rot_dim=rot)
    return rng, table, kp, vp, k64, v64, x, x64, seq, pos, plan, H, kv, n_pages, torch, paged


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page,hd,rot,tokens", [(1, 32, 32, 3), (4, 64, 16, 1), (16, 128, 128, 37), (64, 66, 22, 5),
                                                (1024, 32, 8, 2)])
def test_append_writes_the_pages(dtype, page, hd, rot, tokens):
    (rng, table, kp, vp, k64, v64, x, x64, seq, pos, plan, H, kv, n_pages, torch, paged) = _append_case(
        dtype, page, hd, rot, tokens, page + hd)
    order = rng.permutation(len(pos))                     # rows in any order
    xs, x64, seq, pos = x[torch.from_numpy(order).cuda()], x64[order], seq[order], pos[order]
    q = paged.append(kp, vp, ints(table), ints(pos), xs[:, H:H + kv], xs[:, H + kv:], seq=ints(seq), rotary=plan,
                     q=xs[:, :H])
    freq = ref.frequencies(rot)
    _check(q, x64[:, :H], pos, freq, dtype, rot, False)
    gk, gv = host(kp), host(vp)
    at = [ref.page_of(table, n_pages, page, s, p) for s, p in zip(seq, pos)]
    pages, slots = np.array(at).T
    _check(torch.from_numpy(gk[pages, :, slots]), x64[:, H:H + kv], pos, freq, dtype, rot, False)
    assert np.array_equal(gv[pages, :, slots], x64[:, H + kv:])
    gk[pages, :, slots], gv[pages, :, slots] = k64[pages, :, slots], v64[pages, :, slots]
    assert np.array_equal(gk, k64) and np.array_equal(gv, v64)       # and nothing else


def test_append_leaves_out_rows_without_a_place():
    """Negative positions, sequences outside the table, absent and impossible
    pages, positions past the table: nothing is written for them."""
    (rng, table, kp, vp, k64, v64, x, x64, seq, pos, plan, H, kv, n_pages, torch, paged) = _append_case(
        "bf16", 8, 64, 64, 1, 11)
    table[1, :] = -1
    table[2, :] = [n_pages, n_pages + 1000, -2 ** 31, 2 ** 31 - 1][:1] * table.shape[1]
    cases = [(0, pos[0]), (1, 3), (2, 3), (0, -1), (-1, 2), (4, 2), (3, table.shape[1] * 8), (3, 2 ** 31 - 1), (3, -2 ** 31),
             (3, pos[3])]
    seq, pos = np.array([c[0] for c in cases]), np.array([c[1] for c in cases])
    xs, _ = normal(rng, (len(cases), H + 2 * kv, 64), "bf16")
    q_out = torch.full((len(cases), H, 64), 7.0, dtype=xs.dtype, device="cuda")
    paged.append(kp, vp, ints(table), ints(pos), xs[:, H:H + kv], xs[:, H + kv:], seq=ints(seq), rotary=plan,
                 q=xs[:, :H], q_out=q_out)
    assert (q_out[1:-1] == 7).all() and not (q_out[0] == 7).any() and not (q_out[-1] == 7).any()
    gk, gv = host(kp), host(vp)
    changed = {tuple(i) for i in np.argwhere((gv != v64).any((1, 3)))}
    assert changed == {ref.page_of(table, n_pages, 8, s, p) for s, p in (cases[0], cases[-1])}
    assert {tuple(i) for i in np.argwhere((gk != k64).any((1, 3)))} == changed


def test_append_without_a_plan_copies():
    (rng, table, kp, vp, *_, x, x64, seq, pos, plan, H, kv, n_pages, torch, paged) = _append_case("f32", 4, 32, 32, 2, 12)
    assert paged.append(kp, vp, ints(table), ints(pos), x[:, H:H + kv], x[:, H + kv:], seq=ints(seq)) is None
    pages, slots = np.array([ref.page_of(table, n_pages, 4, s, p) for s, p in zip(seq, pos)]).T
    assert np.array_equal(host(kp)[pages, :, slots], x64[:, H:H + kv])
    assert np.array_equal(host(vp)[pages, :, slots], x64[:, H + kv:])
