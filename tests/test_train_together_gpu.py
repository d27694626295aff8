"""The operators in a row on data of their own (no library's kernels between them): lookup, gradient, norm and
step, over and over, leave the same bits each time; and the norm over as many gradients as a large model has."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402
from paper_2205_14473_amd.state import adamw_list  # noqa: E402


def fit(bits, steps=120, stream=None):
    """A table fitted to another by its rows' squared distances: (first and last mean distance, all that the
    steps changed)."""
    n, vocab, dim, scale = 3000, 211, 72, 2.0
    gen = torch.Generator(device="cuda").manual_seed(8)
    table, aim = (torch.randn((vocab, dim), device="cuda", generator=gen) for _ in range(2))
    start = (table - aim).norm().item()
    grad, x = torch.empty_like(table), torch.empty((n, dim), device="cuda")
    c = E.Embed(tokens=n, vocab=vocab, dim=dim, table_stride=dim, x_stride=dim, padding=-1, scale=scale, index_bits=64)
    ws = torch.empty(E.ea_embed_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    tl = adamw_list([table], [grad], state_bits=bits)
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    norm_ws = torch.empty(E.ea_grad_norm_workspace_bytes(tl), dtype=torch.uint8, device="cuda")
    cfg = E.AdamW(lr=0.05, beta1=0.9, beta2=0.99, eps=1e-8, state_bits=bits, seed=3,
                  rounding=E.EA_ROUND_STOCHASTIC if bits == 8 else E.EA_ROUND_NEAREST)
    norms = []
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        for t in range(1, steps + 1):
            ids = torch.randint(0, vocab, (n,), device="cuda", generator=gen)
            E.ea_embed_lookup(c, table, ids, x)
            E.ea_embed_grad(c, ids, (x - aim[ids] * scale) / n, grad, False, ws)
            E.ea_grad_norm(tl, 1.0, 0.1, norm, factor, norm_ws)
            E.ea_adamw_step(cfg, t, tl, factor)
            norms.append(norm.clone())
    torch.cuda.synchronize()
    return start, (table - aim).norm().item(), [table, torch.cat(norms), *tl.states, *tl.scales]


@pytest.mark.parametrize("bits", [32, 8])
def test_training_leaves_the_same_bits(bits):
    """Every step's norm, and the table and the states at the end, from run to run and on another stream."""
    first, last, held = fit(bits)
    assert last < 0.1 * first                       # 120 steps of 0.05 against distances of about 1.1 an element
    for stream in (None, torch.cuda.Stream()):
        for x, y in zip(fit(bits, stream=stream)[2], held):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))


def test_8_bit_states_fit_as_32_bit_ones():
    a, b = fit(32), fit(8)
    assert a[0] == b[0] and abs(b[1] - a[1]) < 0.05 * a[0]


@pytest.mark.parametrize("sizes", [[(1 << 27) + 70_001], [1 << 27, 5, 9_000_001, 1 << 20], [(1 << 28) + 3, 77]])
def test_norm_of_large_lists(sizes):
    """From 2^27 elements on chunks are longer than 16,384: the ends of the tensors and of the chunks count once."""
    assert sum(sizes) > 8192 * 16384
    flat = torch.zeros(sum(sizes) + 2 * len(sizes), dtype=torch.bfloat16, device="cuda")
    grads, at, terms = [], 1, 0
    for n in sizes:
        g = flat[at:at + n]
        spots = {0, n - 1, n // 2} | {k for c in (16384, 32768, 65536) for k in (c - 1, c, n // c * c - 1, n // c * c) if 0 <= k < n}
        for i, k in enumerate(sorted(spots)):
            g[k] = 1 + i % 5
            terms += (1 + i % 5) ** 2
        grads.append(g)
        at += n + 1
        flat[at - 1] = float("nan")                 # beside the gradients
    flat[0] = float("nan")
    tl = E.TensorList(grads)
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(E.ea_grad_norm_workspace_bytes(tl), dtype=torch.uint8, device="cuda")
    E.ea_grad_norm(tl, 1.0, math.inf, norm, factor, ws)
    assert norm.item() == torch.tensor(math.sqrt(terms), dtype=torch.float32).item()   # integers: exact until the root


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("count", [1, 4, 5, 8, 9, 12])
@pytest.mark.parametrize("total", [60, 4_097, 65_536, 65_537])
def test_norm_of_few_and_many_small_gradients(count, total, kind):
    """On both sides of the limits for one launch; integers, so the sum of squares is exact."""
    sizes = [total // count] * (count - 1)
    sizes.append(total - sum(sizes))
    gen = torch.Generator().manual_seed(total + count)
    grads = [torch.randint(-4, 5, (n,), generator=gen).to(kind).cuda() for n in sizes] + [torch.empty(0, dtype=kind, device="cuda")]
    want = math.sqrt(sum(int((g.double() ** 2).sum().item()) for g in grads))
    tl = E.TensorList(grads)
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    ws = torch.empty(E.ea_grad_norm_workspace_bytes(tl), dtype=torch.uint8, device="cuda")
    E.ea_grad_norm(tl, 1.0, math.inf, norm, factor, ws)
    assert norm.item() == torch.tensor(want, dtype=torch.float32).item() and factor.item() == 1.0
