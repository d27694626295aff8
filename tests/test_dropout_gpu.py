"""Dropout and its gradient, bit for bit against the draws of the generator: types, rates, odd and strided rows, in
place, dropped infinities and NaN, steps read on the device, elements past 2^32."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402
import paper_2205_14473_amd as E  # noqa: E402
from layer_util import TYPES  # noqa: E402

SEED = 0x0123456789ABCDEF


def config(rows, dim, x, y, p=0.1, xgap=0, ygap=0, site=3, seed=SEED):
    return E.Dropout(rows=rows, dim=dim, x_stride=dim + xgap, y_stride=dim + ygap, p=p, x_type=E.ea_type(x),
                     y_type=E.ea_type(y), site=site, seed=seed)


def same(a, b):
    return torch.equal(a.cpu().contiguous().view(torch.uint8), b.cpu().contiguous().view(torch.uint8))


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("rows,dim,xgap,ygap,shift", [(1, 1, 0, 0, 0), (1, 8, 0, 0, 0), (3, 5, 0, 0, 1), (7, 1, 2, 3, 1), (5, 3, 1, 0, 0),
                                                      (4, 8, 8, 0, 0), (9, 17, 0, 4, 1), (33, 64, 0, 0, 0), (1, 5000, 3, 3, 1),
                                                      (257, 1001, 0, 0, 0), (64, 1001, 7, 0, 1), (300, 768, 0, 0, 0), (2, 70_000, 0, 1, 0)])
@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f16")])
def test_forward_and_gradient(rows, dim, xgap, ygap, shift, x, y, residual):
    xt, yt = TYPES[x], TYPES[y]
    gen = torch.Generator().manual_seed(rows + dim)
    xv, rv, dv = (torch.randn((rows, dim), generator=gen).to(t) for t in (xt, yt, yt))
    c = config(rows, dim, xt, yt, 0.3, xgap, ygap)
    keep, factor = L.kept(SEED, 77, 3, rows, dim, 0.3)
    _, xd = L.spaced(xv, dim + xgap, xt, shift)
    _, rd = L.spaced(rv, dim + ygap, yt, shift)
    yf, yd = L.spaced((rows, dim), dim + ygap, yt, shift)
    E.ea_dropout(c, 77, xd, rd if residual else None, yd)
    assert same(yd, L.dropout(xv, rv if residual else None, keep, factor, yt))
    assert L.guards_kept(yf, yd, shift)
    if residual:
        E.ea_dropout(c, 77, xd, rd, rd)
        assert same(rd, yd)
    _, dd = L.spaced(dv, dim + ygap, yt, shift)
    df, dx = L.spaced((rows, dim), dim + xgap, xt, shift)
    E.ea_dropout_grad(c, 77, dd, dx)
    assert same(dx, L.dropout(dv, None, keep, factor, xt))
    assert L.guards_kept(df, dx, shift)


@pytest.mark.parametrize("x", TYPES)
@pytest.mark.parametrize("y", TYPES)
def test_types(x, y):
    gen = torch.Generator().manual_seed(9)
    xv, rv = torch.randn((21, 67), generator=gen).to(TYPES[x]), torch.randn((21, 67), generator=gen).to(TYPES[y])
    keep, factor = L.kept(SEED, 5, 3, 21, 67, 0.1)
    out = torch.empty((21, 67), dtype=TYPES[y], device="cuda")
    E.ea_dropout(config(21, 67, TYPES[x], TYPES[y]), 5, xv.cuda(), rv.cuda(), out)
    assert same(out, L.dropout(xv, rv, keep, factor, TYPES[y]))


@pytest.mark.parametrize("p", [0.0, 2.0 ** -17, 2.0 ** -16, 0.05, 0.5, 0.9, 1 - 2.0 ** -16, 1 - 2.0 ** -17, 1.0])
def test_rates_and_values_that_are_dropped(p):
    rows, dim = 130, 513
    xv = torch.randn((rows, dim), generator=torch.Generator().manual_seed(1))
    keep, factor = L.kept(SEED, 0, 3, rows, dim, p)
    xv[~keep] = torch.tensor([float("nan"), float("inf"), -float("inf")]).repeat(rows * dim)[:int((~keep).sum())]
    out = torch.empty((rows, dim), device="cuda")
    E.ea_dropout(config(rows, dim, torch.float32, torch.float32, p), 0, xv.cuda(), None, out)
    assert same(out, L.dropout(xv, None, keep, factor, torch.float32)) and not out.isnan().any()
    share = 1 - keep.double().mean().item()
    assert abs(share - p) <= 5 * (p * (1 - p) / (rows * dim)) ** 0.5 + 2.0 ** -17


def test_sites_steps_and_seeds_draw_differently():
    n, keeps = 100_000, []
    x = torch.ones((1, n), device="cuda")
    out = torch.empty_like(x)
    for site, t, seed in ((0, 1, SEED), (1, 1, SEED), (0, 2, SEED), (0, 1, SEED + 1), (0, 1, SEED + (1 << 32)),
                          (2 ** 32 - 1, 2 ** 32 - 1, 2 ** 64 - 1)):
        E.ea_dropout(config(1, n, torch.float32, torch.float32, 0.5, site=site, seed=seed), t, x, None, out)
        keep, _ = L.kept(seed, t, site, 1, n, 0.5)
        assert torch.equal(out.cpu() != 0, keep)
        keeps.append(out.cpu() != 0)
    for i, a in enumerate(keeps):
        for b in keeps[:i]:
            # shares of agreement of independent halves: 0.5, five deviations of 0.5 / sqrt(n)
            assert abs((a == b).double().mean().item() - 0.5) < 2.5 / n ** 0.5


def test_average_is_the_input():
    """The factor makes up for the share that is kept: sums over many draws, five deviations."""
    n, p = 1 << 20, 0.1
    x, out = torch.ones((1, n), device="cuda"), torch.empty((1, n), device="cuda")
    E.ea_dropout(config(1, n, torch.float32, torch.float32, p), 11, x, None, out)
    assert abs(out.double().mean().item() - 1) < 5 * (p / (1 - p) / n) ** 0.5


def test_step_on_the_device_and_in_a_graph():
    rows, dim = 50, 203
    c = config(rows, dim, torch.bfloat16, torch.bfloat16)
    xv = torch.randn((rows, dim), generator=torch.Generator().manual_seed(1)).bfloat16()
    x, out, dx = xv.cuda(), torch.zeros_like(xv.cuda()), torch.zeros_like(xv.cuda())
    t = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E.ea_dropout(c, 0, x, x, out, t_dev=t)
        E.ea_dropout_grad(c, 0, x, dx, t_dev=t)
    for k in (3, 4, 2 ** 31 - 1):
        t.fill_(k)
        graph.replay()
        torch.cuda.synchronize()
        keep, factor = L.kept(SEED, k, 3, rows, dim, 0.1)
        assert same(out, L.dropout(xv, xv, keep, factor, torch.bfloat16))
        assert same(dx, L.dropout(xv, None, keep, factor, torch.bfloat16)) and t.item() == k
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    E.ea_dropout(c, 3, x, None, out, stream=s)
    s.synchronize()
    keep, factor = L.kept(SEED, 3, 3, rows, dim, 0.1)
    assert same(out, L.dropout(xv, None, keep, factor, torch.bfloat16))


@pytest.mark.parametrize("gap", [0, 2])
def test_elements_past_32_bits(gap):
    """The last of more than 2^32 elements: their numbers and their offsets."""
    dim = (1 << 22) + 5
    rows = (1 << 32) // dim + 3
    stride = dim + gap
    x = torch.empty(rows * stride, dtype=torch.bfloat16, device="cuda").fill_(1.0)
    x = torch.as_strided(x, (rows, dim), (stride, 1))
    c = config(rows, dim, torch.bfloat16, torch.bfloat16, 0.25, gap, gap)
    E.ea_dropout(c, 9, x, None, x)
    keep = last_kept(rows, dim, 4096, 9, 0.25)
    assert torch.equal(x[-1, -4096:].cpu() != 0, keep)


def last_kept(rows, dim, count, t, p):
    import numpy as np
    import train_util as R
    n = rows * dim
    first = (n - count) // 8
    words = R.philox_words(SEED, t, 3, (n - first * 8 + 7) // 8 * 4, first=first)
    halves = np.stack([words & np.uint32(0xFFFF), words >> np.uint32(16)], 1).reshape(-1)
    at = n - count - first * 8
    return torch.from_numpy(halves[at:at + count].astype(np.int64) >= int(p * 65536))


def test_no_rows():
    c = config(0, 5, torch.float32, torch.float32)
    none = torch.empty((0, 5), device="cuda")
    E.ea_dropout(c, 1, none, None, none)
    E.ea_dropout_grad(c, 1, none, none)
