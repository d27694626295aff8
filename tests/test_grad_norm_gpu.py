"""The global gradient norm and the clip factor against 64 bits: types, sizes, alignment, overflow,
gradients that are not finite, and the step that takes the factor."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402
from paper_2205_14473_amd.state import adamw_list  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def norm_of(grads, scale=1.0, max_norm=math.inf, stream=None):
    tl = E.TensorList(grads)
    norm, factor = torch.full((1,), 7.0, device="cuda"), torch.full((1,), 7.0, device="cuda")
    need = E.ea_grad_norm_workspace_bytes(tl)
    big = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    E.ea_grad_norm(tl, scale, max_norm, norm, factor, big[:need] if need else None, stream)
    torch.cuda.synchronize()
    assert bool((big[need:] == 0xA5).all()), "a write past the workspace"
    return norm.item(), factor.item()


def want(grads, scale=1.0):
    return float(np.float32(scale)) * math.sqrt(sum(float((g.cpu().double() ** 2).sum()) for g in grads))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("sizes", [[1], [3, 0, 2], [255, 256, 257], [4096], [4097, 1, 8191], [1_000_003],
                                   list(range(1, 400))])
def test_norm(kind, sizes):
    gen = torch.Generator().manual_seed(len(sizes))
    flat = (torch.randn(sum(sizes) + len(sizes), generator=gen) * 0.1).to(TYPES[kind]).cuda()
    grads, at = [], 1                               # one element apart: most start off alignment
    for n in sizes:
        grads.append(flat[at:at + n])
        at += n + 1 if at + n + 1 <= flat.numel() else n
    norm, factor = norm_of(grads, 0.5, 0.25)
    w = want(grads, 0.5)
    # one rounding to binary32 of a binary64 sum
    assert abs(norm - w) <= 2.0 ** -23 * w
    f = 0.5 * min(1.0, 0.25 / w)
    assert abs(factor - f) <= 2.0 ** -22 * f


def test_large_and_small_values_neither_overflow_nor_vanish():
    for size in (1e30, 1e-30, 3e38, 1e-42):
        g = [torch.full((5000,), size, device="cuda")]
        norm, factor = norm_of(g)
        w = want(g)
        assert (norm == math.inf and math.isnan(factor)) if w > 3.4e38 else abs(norm - w) <= 2.0 ** -23 * w + 1e-45


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_not_finite(bad):
    g = [torch.zeros(5000, device="cuda"), torch.zeros(100, device="cuda")]
    g[1][99] = bad
    norm, factor = norm_of(g, max_norm=1.0)
    assert not math.isfinite(norm) and math.isnan(factor)
    # the step with that factor is skipped
    p = [torch.ones_like(x) for x in g]
    tl = adamw_list(p, g)
    cfg = E.AdamW(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, state_bits=32)
    E.ea_adamw_step(cfg, 1, tl, torch.full((1,), factor, device="cuda"))
    assert all(bool((x == 1).all()) for x in p) and not any(s.any() for s in tl.states)


def test_no_clipping_and_no_gradients():
    g = [torch.full((16,), 0.25, device="cuda")]
    assert norm_of(g) == (1.0, 1.0)
    assert norm_of(g, 2.0, 2.0) == (2.0, 2.0)       # a norm of max_norm is not clipped
    assert norm_of([torch.zeros(9, device="cuda")], 3.0, 1.0) == (0.0, 3.0)
    assert norm_of([], 3.0, 1.0) == (0.0, 3.0)
    assert norm_of([torch.empty(0, device="cuda")], 3.0, 1.0) == (0.0, 3.0)


def test_same_bits_every_time_and_on_another_stream():
    g = [torch.randn(3_000_001, device="cuda"), torch.randn(5, device="cuda")]
    first = norm_of(g, 1.0, 1.0)
    assert all(norm_of(g, 1.0, 1.0, s) == first for s in (None, torch.cuda.Stream(), None))


def test_norm_and_step_in_a_graph():
    """Norm, factor and step captured together; each replay on new gradients against eager calls."""
    g, e = (torch.empty(70_000, device="cuda") for _ in range(2))
    p, q = torch.ones(70_000, device="cuda"), torch.ones(70_000, device="cuda")
    la, lb = adamw_list([p], [g]), adamw_list([q], [e])
    cfg = E.AdamW(lr=0.01, beta1=0.9, beta2=0.99, eps=1e-8, state_bits=32)
    bufs = [[torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda"),
             torch.empty(E.ea_grad_norm_workspace_bytes(la), dtype=torch.uint8, device="cuda")] for _ in range(2)]
    t_dev = torch.ones(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        E.ea_grad_norm(la, 1.0, 1.0, *bufs[0])
        E.ea_adamw_step_scheduled(cfg, E.Schedule(kind=E.EA_SCHED_CONSTANT), t_dev, la, bufs[0][1])
    for t in range(1, 5):
        g.copy_(torch.randn(70_000, generator=torch.Generator().manual_seed(t)))
        if t == 3:
            g[5] = math.nan
        e.copy_(g)
        graph.replay()
        E.ea_grad_norm(lb, 1.0, 1.0, *bufs[1])
        E.ea_adamw_step(cfg, t, lb, bufs[1][1])
        torch.cuda.synchronize()
        assert torch.equal(p, q) and all(torch.equal(x, y) for x, y in zip(la.states, lb.states)), f"step {t}"
    assert torch.isfinite(p).all()


def test_what_stands_beside_the_gradients_is_not_read():
    for sizes in ([1, 5, 300], [70_001, 9]):
        flat = torch.full((sum(sizes) + 8,), float("nan"), device="cuda")
        grads, at = [], 3
        for n in sizes:
            grads.append(flat[at:at + n])
            at += n + 1
        for g in grads:
            g.fill_(0.5)
        norm, _ = norm_of(grads)
        assert abs(norm - want(grads)) <= 2.0 ** -23 * norm
