"""The binding records nothing for autograd, and refuses what would lose a
gradient: on the host, before it looks at anything else."""
import pytest

from paper_2606_29223_amd import dexlib, paged

torch = pytest.importorskip("torch")
from torch.autograd import forward_ad  # noqa: E402

CALLS = {
    "rope": (lambda p, n, t, **x: paged.rope(p, n, x["q"], x["k"], x["q_out"], x["k_out"]), "q k q_out k_out"),
    "append": (lambda p, n, t, **x: paged.append(x["k_pages"], x["v_pages"], t, n, x["k"], x["v"], rotary=p, q=x["q"],
                                                 q_out=x["q_out"]), "q k v k_pages v_pages q_out"),
    "attention": (lambda p, n, t, **x: paged.attention(x["q"], x["k_pages"], x["v_pages"], t, n, out=x["out"]),
                  "q k_pages v_pages out"),
    "copy": (lambda p, n, t, **x: paged.copy(x["k_pages"][None], x["v_pages"][None], n, n), "k_pages v_pages"),
    "beam_select": (lambda p, n, t, **x: paged.beam_select(x["logits"], x["scores"]), "logits scores"),
}
WHICH = [(call, name) for call, (_, names) in CALLS.items() for name in names.split()]


def _arguments(device):
    x = {n: torch.zeros((2, 2, 32), device=device) for n in ("q", "k", "v", "q_out", "k_out", "out")}
    x.update({n: torch.zeros((4, 2, 4, 32), device=device) for n in ("k_pages", "v_pages")})
    x.update(logits=torch.zeros((4, 9), device=device), scores=torch.zeros((2, 2), device=device))
    plan = paged.Rotary(32, device=device)
    return plan, torch.zeros(2, dtype=torch.int32, device=device), torch.zeros((2, 2), dtype=torch.int32, device=device), x


@pytest.fixture(scope="module", autouse=True)
def _built():
    import os
    if not os.path.exists(dexlib.LIB_PATH):
        pytest.skip("libdex.so not built")


@pytest.mark.parametrize("call,name", WHICH)
def test_a_tensor_that_requires_grad_is_refused(call, name):
    p, n, t, x = _arguments("cpu")
    x[name].requires_grad_()
    with pytest.raises(dexlib.DexError, match="requires grad"):
        CALLS[call][0](p, n, t, **x)
    with torch.no_grad(), pytest.raises(dexlib.DexError, match="not on a GPU"):
        CALLS[call][0](p, n, t, **x)


@pytest.mark.parametrize("call,name", WHICH)
def test_a_tangent_is_refused(call, name):
    p, n, t, x = _arguments("cpu")
    with forward_ad.dual_level():
        x[name] = forward_ad.make_dual(x[name], torch.ones_like(x[name]))
        with pytest.raises(dexlib.DexError, match="tangent"):
            CALLS[call][0](p, n, t, **x)


@pytest.mark.gpu
@pytest.mark.parametrize("call", CALLS)
def test_without_grad_mode_the_calls_run(call):
    p, n, t, x = _arguments("cuda")
    for v in x.values():
        v.requires_grad_()
    with torch.no_grad():
        got = CALLS[call][0](p, n, t, **x)
    for v in x.values():
        v.requires_grad_(False)
    with forward_ad.dual_level():                         # a level without tangents takes nothing away
        again = CALLS[call][0](p, n, t, **x)
    flat = lambda r: [] if r is None else [r] if torch.is_tensor(r) else list(r)
    assert all(torch.equal(a, b) for a, b in zip(flat(got), flat(again)))
