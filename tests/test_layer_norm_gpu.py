"""Layer norm and its gradient against 64 bits: types, widths of every form, odd widths, row gaps, misaligned rows,
missing weights, accumulation, in place, rows of one value, infinities and NaN, other streams, graphs."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402
import paper_2205_14473_amd as E  # noqa: E402
import train_util as R  # noqa: E402
from layer_util import TYPES  # noqa: E402

EPS = 1e-5


def config(rows, dim, x, y, w=torch.float32, xgap=0, ygap=0, eps=EPS):
    return E.LayerNorm(rows=rows, dim=dim, x_stride=dim + xgap, y_stride=dim + ygap, eps=eps, x_type=E.ea_type(x),
                       y_type=E.ea_type(y), w_type=E.ea_type(w))


def inputs(rows, dim, x, y, w, seed=0, offset=0.3):
    gen = torch.Generator().manual_seed(seed + rows * 7919 + dim)
    size = torch.exp(0.7 * torch.randn(dim, generator=gen))
    xv = (torch.randn((rows, dim), generator=gen) * size + offset).to(x)
    wv, bv = (1 + 0.1 * torch.randn(dim, generator=gen)).to(w), (0.1 * torch.randn(dim, generator=gen)).to(w)
    dy = (torch.randn((rows, dim), generator=gen) * 1e-2).to(y)
    add = (torch.randn((rows, dim), generator=gen) * 1e-2).to(x)
    return xv, wv, bv, dy, add


SHAPES = [(1, 1), (3, 2), (7, 7), (5, 64), (9, 255), (4, 256), (33, 257), (6, 512), (5, 513), (17, 768), (1030, 40),
          (3, 1000), (16, 1024), (3, 1025), (4, 2049), (2, 3001), (3, 4096), (2, 4097), (1, 8193), (2, 12_289), (1, 16_384),
          (2, 16_385), (3, 20_000), (1, 70_001), (9001, 8), (2500, 130)]


@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("f16", "f32"), ("f32", "bf16")])
def test_forward(rows, dim, x, y):
    xt, yt = TYPES[x], TYPES[y]
    xv, wv, bv, _, _ = inputs(rows, dim, xt, yt, torch.float32)
    gap, shift = (0, 0) if dim % 2 == 0 else (3, 1)
    _, xd = L.spaced(xv, dim + gap, xt, shift)
    yf, yd = L.spaced((rows, dim), dim + 2 * gap, yt, shift)
    mean, rstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    E.ea_layer_norm(config(rows, dim, xt, yt, xgap=gap, ygap=2 * gap), xd, wv.cuda(), bv.cuda(), yd, mean, rstd)
    want = L.Norm(xv.double(), wv.double(), bv.double(), EPS)
    R.within(mean, want.mean, want.mean_bound, "mean")
    R.within(rstd, want.rstd, want.rstd_bound, "rstd")
    R.within(yd, want.y, want.y_bound + L.rounding(want.y, yt), "y")
    assert L.guards_kept(yf, yd, shift)


@pytest.mark.parametrize("w", TYPES)
@pytest.mark.parametrize("x", TYPES)
@pytest.mark.parametrize("y", TYPES)
@pytest.mark.parametrize("dim", [96, 1301])
def test_types(dim, x, y, w):
    rows, xt, yt, wt = 37, TYPES[x], TYPES[y], TYPES[w]
    xv, wv, bv, dy, add = inputs(rows, dim, xt, yt, wt)
    c = config(rows, dim, xt, yt, wt)
    yd = torch.empty((rows, dim), dtype=yt, device="cuda")
    E.ea_layer_norm(c, xv.cuda(), wv.cuda(), bv.cuda(), yd)
    want = L.Norm(xv.double(), wv.double(), bv.double(), EPS)
    R.within(yd, want.y, want.y_bound + L.rounding(want.y, yt), "y")
    check_grad(c, xv, dy, wv, add, wv, bv, want)
    check_grad(c, xv, dy, wv, None, None, None, want)


def check_grad(c, xv, dy, wv, add, dw, db, want, shift=0, in_place=None):
    """Runs the gradient and checks all that it writes; dw and db: accumulate to these."""
    rows, dim = xv.shape
    xt, yt, wt = xv.dtype, dy.dtype, wv.dtype
    mean, rstd = want.mean.float(), want.rstd.float()
    _, xd = L.spaced(xv, c.x_stride, xt, shift)
    _, dyd = L.spaced(dy, c.y_stride, yt, shift)
    addd = None if add is None else L.spaced(add, c.x_stride, xt, shift)[1]
    flat, dx = L.spaced((rows, dim), c.x_stride, xt, shift)
    if in_place == "add":
        dx = addd
    elif in_place == "x":
        dx = xd
    elif in_place == "dy":
        dx = dyd
    dwd, dbd = (torch.full((dim + 2,), L.GUARD, dtype=wt, device="cuda") for _ in range(2))
    if dw is not None:
        dwd[1:-1], dbd[1:-1] = dw.cuda(), db.cuda()
    need = E.ea_layer_norm_workspace_bytes(c)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    E.ea_layer_norm_grad(c, xd, dyd, wv.cuda(), mean.cuda(), rstd.cuda(), addd, dx, dwd[1:-1], dbd[1:-1], dw is not None,
                         ws[:need] if need else None)
    torch.cuda.synchronize()
    got = L.NormGrad(xv.double(), dy.double(), wv.double(), mean.double(), rstd.double(),
                     None if add is None else add.double(), *(None if v is None else v.double() for v in (dw, db)))
    R.within(dx, got.dx, got.dx_bound + L.rounding(got.dx, xt), "dx")
    R.within(dwd[1:-1], got.dw, got.dw_bound + L.rounding(got.dw, wt), "dweight")
    R.within(dbd[1:-1], got.db, got.db_bound + L.rounding(got.db, wt), "dbias")
    assert bool((ws[need:] == 0xA5).all()), "a write past the workspace"
    assert all(bool(v[k] == L.GUARD) for v in (dwd, dbd) for k in (0, -1))
    assert in_place or L.guards_kept(flat, dx, shift)
    return dx, dwd, dbd


@pytest.mark.parametrize("rows,dim", SHAPES)
@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_gradient(rows, dim, x, y):
    xt, yt = TYPES[x], TYPES[y]
    xv, wv, bv, dy, add = inputs(rows, dim, xt, yt, torch.float32, seed=1)
    gap, shift = (0, 0) if dim % 2 == 0 else (3, 1)
    c = config(rows, dim, xt, yt, xgap=gap, ygap=2 * gap)
    want = L.Norm(xv.double(), wv.double(), bv.double(), EPS)
    check_grad(c, xv, dy, wv, add if rows % 2 else None, *((wv, bv) if rows % 3 else (None, None)), want, shift)


@pytest.mark.parametrize("where", ["add", "x", "dy"])
@pytest.mark.parametrize("rows,dim", [(70, 300), (3, 5000), (2, 20_001)])
def test_gradient_in_place(rows, dim, where):
    xv, wv, bv, dy, add = inputs(rows, dim, torch.float32, torch.float32, torch.float32, seed=2)
    want = L.Norm(xv.double(), wv.double(), bv.double(), EPS)
    check_grad(config(rows, dim, torch.float32, torch.float32), xv, dy, wv, add, None, None, want, in_place=where)


@pytest.mark.parametrize("dim", [100, 5000, 20_001])
def test_forward_in_place_and_without_weights(dim):
    xv, wv, bv, _, _ = inputs(11, dim, torch.bfloat16, torch.bfloat16, torch.float32)
    c, x, y = config(11, dim, torch.bfloat16, torch.bfloat16), xv.cuda(), torch.empty((11, dim), dtype=torch.bfloat16, device="cuda")
    E.ea_layer_norm(c, x, wv.cuda(), bv.cuda(), y)
    E.ea_layer_norm(c, x, wv.cuda(), bv.cuda(), x)
    assert torch.equal(x, y)
    E.ea_layer_norm(c, xv.cuda(), None, None, y)
    one = torch.ones(dim, dtype=torch.float64)
    want = L.Norm(xv.double(), one, 0 * one, EPS)
    R.within(y, want.y, want.y_bound + L.rounding(want.y, torch.bfloat16), "y")
    dx, dw = torch.empty_like(y), torch.empty(dim, device="cuda")
    ws = torch.empty(E.ea_layer_norm_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    mean, rstd = want.mean.float(), want.rstd.float()
    got = L.NormGrad(xv.double(), y.cpu().double(), one, mean.double(), rstd.double())
    for weights in ((dw, None), (None, dw), (None, None)):
        E.ea_layer_norm_grad(c, xv.cuda(), y, None, mean.cuda(), rstd.cuda(), None, dx, *weights, False,
                             ws if weights[0] is not None or weights[1] is not None else None)
        R.within(dx, got.dx, got.dx_bound + L.rounding(got.dx, torch.bfloat16), "dx")
        if weights[0] is not None:
            R.within(dw, got.dw, got.dw_bound, "dweight")
        elif weights[1] is not None:
            R.within(dw, got.db, got.db_bound, "dbias")


@pytest.mark.parametrize("dim", [33, 1024, 5000, 17_000])
def test_rows_of_one_value_and_far_from_zero(dim):
    """A row of one value: the deviations are the mean's rounding, and eps keeps the quotient small.  Offsets of a
    thousand deviations: the two-pass sums keep the variance."""
    xv = torch.full((4, dim), 3.0)
    xv[1] = 0.0
    xv[2:] = torch.randn((2, dim), generator=torch.Generator().manual_seed(dim)) + 1000.0
    one = torch.ones(dim)
    y, mean, rstd = torch.empty((4, dim), device="cuda"), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    E.ea_layer_norm(config(4, dim, torch.float32, torch.float32), xv.cuda(), one.cuda(), 0 * one.cuda(), y, mean, rstd)
    want = L.Norm(xv.double(), one.double(), 0 * one.double(), EPS)
    R.within(y, want.y, want.y_bound, "y")
    R.within(rstd, want.rstd, want.rstd_bound, "rstd")
    assert bool((y[1] == 0).all())


@pytest.mark.parametrize("dim", [70, 3000, 17_000])
def test_infinities_and_nan_stay_in_their_rows(dim):
    xv, wv, bv, dy, _ = inputs(9, dim, torch.float32, torch.float32, torch.float32)
    good = [0, 2, 3, 5, 6, 8]
    bad = xv.clone()
    bad[1, dim // 2], bad[4, 0], bad[7, dim - 1] = float("nan"), float("inf"), 1e30
    c, out = config(9, dim, torch.float32, torch.float32), []
    for v in (xv, bad):
        y, mean, rstd = torch.empty((9, dim), device="cuda"), torch.empty(9, device="cuda"), torch.empty(9, device="cuda")
        E.ea_layer_norm(c, v.cuda(), wv.cuda(), bv.cuda(), y, mean, rstd)
        dx = torch.empty_like(y)
        E.ea_layer_norm_grad(c, v.cuda(), dy.cuda(), wv.cuda(), mean, rstd, None, dx, None, None, False, None)
        out.append((y, mean, rstd, dx))
    for a, b in zip(*out):
        assert torch.equal(a[good], b[good])
    assert out[1][0][1].isnan().all() and out[1][0][4].isnan().all()


@pytest.mark.parametrize("accumulate", [False, True])
def test_no_rows(accumulate):
    c = config(0, 50, torch.float32, torch.float32)
    assert E.ea_layer_norm_workspace_bytes(c) == 0
    none = torch.empty((0, 50), device="cuda")
    dw, db = torch.full((50,), 2.0, device="cuda"), torch.full((50,), 3.0, device="cuda")
    E.ea_layer_norm(c, none, dw, db, none)
    E.ea_layer_norm_grad(c, none, none, dw.clone(), torch.empty(0, device="cuda"), torch.empty(0, device="cuda"), None,
                         none, dw, db, accumulate, None)
    assert bool((dw == (2.0 if accumulate else 0.0)).all()) and bool((db == (3.0 if accumulate else 0.0)).all())


def test_gradient_by_differences():
    """Along random directions of x, weight and bias, by the 64-bit norm: central differences of a step of 2^-12 are off
    by their third-order term, 2^-24 of the function's scale of 1."""
    rows, dim = 6, 90
    xv, wv, bv, dy, _ = inputs(rows, dim, torch.float32, torch.float32, torch.float32, seed=5)
    dy = dy * 100
    c = config(rows, dim, torch.float32, torch.float32)
    y, mean, rstd = torch.empty((rows, dim), device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    E.ea_layer_norm(c, xv.cuda(), wv.cuda(), bv.cuda(), y, mean, rstd)
    dx, dw, db = torch.empty_like(y), torch.empty(dim, device="cuda"), torch.empty(dim, device="cuda")
    ws = torch.empty(E.ea_layer_norm_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    E.ea_layer_norm_grad(c, xv.cuda(), dy.cuda(), wv.cuda(), mean, rstd, None, dx, dw, db, False, ws)
    f = lambda p: (L.Norm(*p, EPS).y * dy.double()).sum().item()  # noqa: E731
    at, h = [v.double() for v in (xv, wv, bv)], 2.0 ** -12
    for k, got in enumerate((dx, dw, db)):
        D = torch.randn(at[k].shape, dtype=torch.float64, generator=torch.Generator().manual_seed(k))
        side = [f([v + s * h * D if i == k else v for i, v in enumerate(at)]) for s in (1, -1)]
        slope, want = (side[0] - side[1]) / (2 * h), (got.cpu().double() * D).sum().item()
        assert abs(slope - want) <= 1e-5 * (got.cpu().double() * D).abs().sum().item() + 1e-5


def test_rows_past_32_bit_offsets():
    """Two rows whose second one starts past 2^31 elements."""
    stride = (1 << 31) + 10
    flat = torch.zeros(stride + 70, dtype=torch.bfloat16, device="cuda")
    x = torch.as_strided(flat, (2, 70), (stride, 1))
    xv = torch.randn((2, 70), generator=torch.Generator().manual_seed(0)).bfloat16()
    x.copy_(xv)
    one = torch.ones(70)
    c = E.LayerNorm(rows=2, dim=70, x_stride=stride, y_stride=70, eps=EPS, x_type=E.EA_BF16, y_type=E.EA_F32)
    y = torch.empty((2, 70), device="cuda")
    E.ea_layer_norm(c, x, one.cuda(), None, y)
    want = L.Norm(xv.double(), one.double(), 0 * one.double(), EPS)
    R.within(y, want.y, want.y_bound, "y")


def test_graph_streams_and_the_same_bits():
    rows, dim = 3001, 520
    xv, wv, bv, dy, _ = inputs(rows, dim, torch.bfloat16, torch.bfloat16, torch.float32)
    c = config(rows, dim, torch.bfloat16, torch.bfloat16)
    x, d, w, b = xv.cuda(), dy.cuda(), wv.cuda(), bv.cuda()
    ws = torch.empty(E.ea_layer_norm_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    outs = [torch.zeros((rows, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    flat = [torch.zeros(n, device="cuda") for n in (rows, rows, dim, dim)]

    def both(stream=None):
        E.ea_layer_norm(c, x, w, b, outs[0], flat[0], flat[1], stream=stream)
        E.ea_layer_norm_grad(c, x, d, w, flat[0], flat[1], None, outs[1], flat[2], flat[3], False, ws, stream=stream)

    both()
    torch.cuda.synchronize()
    held = [t.clone() for t in outs + flat]
    s = torch.cuda.Stream()
    both(s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, outs + flat))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for k in range(3):
        x.copy_(xv * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs + flat]
        both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs + flat))
