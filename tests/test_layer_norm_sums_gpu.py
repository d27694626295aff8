"""The weights' gradient of layer norm over many rows, in whole numbers: with a mean of 0 and an rstd of 1, dweight is the sum
over the rows of dy x and dbias that of dy, all partial sums stay far under 2^24, and so every result is exact in any
order: a row that is lost or taken twice shows.  More rows than a launch has workgroups, for every form, with an uneven last
turn or run.  Rows whose squares overflow."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402
import paper_2205_14473_amd as E  # noqa: E402
from layer_util import TYPES  # noqa: E402


def config(rows, dim, x, y, w=torch.float32, xgap=0, ygap=0):
    return E.LayerNorm(rows=rows, dim=dim, x_stride=dim + xgap, y_stride=dim + ygap, eps=1e-5, x_type=E.ea_type(x),
                       y_type=E.ea_type(y), w_type=E.ea_type(w))


def whole(shape, most, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, device="cuda", generator=gen)


def check(rows, dim, x, y, accumulate, gap=0, shift=0):
    """Terms of at most 9 in magnitude over at most 530,000 rows: sums under 2^23."""
    xt, yt = TYPES[x], TYPES[y]
    xv, dy = whole((rows, dim), 3, rows), whole((rows, dim), 3, dim)
    c = config(rows, dim, xt, yt, xgap=gap, ygap=2 * gap)
    xd, dyd = L.spaced(xv.to(xt), c.x_stride, xt, shift)[1], L.spaced(dy.to(yt), c.y_stride, yt, shift)[1]
    flat, dx = L.spaced((rows, dim), c.x_stride, xt, shift)
    w, b = whole((dim,), 1000, 1), whole((dim,), 1000, 2)
    dw, db = (v.float() if accumulate else torch.full((dim,), float("nan"), device="cuda") for v in (w, b))
    need = E.ea_layer_norm_workspace_bytes(c)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    E.ea_layer_norm_grad(c, xd, dyd, None, mean, rstd, None, dx, dw, db, accumulate, ws[:need])
    one = 1 if accumulate else 0
    assert torch.equal(dw.long(), (dy * xv).sum(0) + one * w)
    assert torch.equal(db.long(), dy.sum(0) + one * b)
    assert bool((ws[need:] == 0xFF).all()) and L.guards_kept(flat, dx, shift)


# rows over the workgroups of a launch (256 to 1,024; four rows each of one wave; runs of long rows: 64 of them at most)
SHAPES = [(4097, 8), (9001, 8), (13_003, 130), (5000, 257), (4500, 1001), (5003, 1024),      # one wave
          (1025, 1030), (2500, 1030), (1100, 4096), (2051, 2048), (1700, 3001),            # 4 waves
          (257, 4097), (700, 4100), (600, 8192), (515, 12_289), (523, 16_384),             # 16 waves
          (16, 16_390), (17, 16_390), (37, 16_390), (1025, 16_400), (1100, 16_400), (190, 40_001)]     # not held


@pytest.mark.parametrize("x,y", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("rows,dim", SHAPES)
def test_sums_over_rows(rows, dim, x, y):
    gap, shift = (0, 0) if dim % 2 == 0 else (3, 1)
    check(rows, dim, x, y, rows % 2 == 1, gap, shift)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("dim", [64, 1001, 4096, 8190, 20_001])
def test_sums_beside_results_past_the_caches(dim, kind):
    size = torch.empty(0, dtype=TYPES[kind]).element_size()
    check((64 << 20) // (dim * size) + 3, dim, kind, kind, False)


@pytest.mark.parametrize("dim", [70, 3000, 9000, 17_000])
def test_rows_whose_squares_overflow(dim):
    """The deviation's reciprocal is 0, the row's result the bias, its gradient 0."""
    x = torch.randn((3, dim), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    x[1, dim - 1] = 1e30
    w, b = torch.randn(dim, device="cuda"), torch.randn(dim, device="cuda")
    y, dx, mean, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(3, device="cuda"), torch.empty(3, device="cuda")
    c = config(3, dim, torch.float32, torch.float32)
    E.ea_layer_norm(c, x, w, b, y, mean, rstd)
    E.ea_layer_norm_grad(c, x, torch.randn_like(x), w, mean, rstd, None, dx, None, None, False, None)
    assert rstd[1].item() == 0 and torch.equal(y[1], b) and bool((dx[1] == 0).all())
    assert bool((rstd[::2] > 0).all()) and bool(dx[::2].isfinite().all())
