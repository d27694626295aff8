"""Layer norm's means are quotients, not products with a rounded 1 / dim: where a row's sum is exact, a whole multiple of
the row's width, so is its mean, and what is left of the row after its subtraction is 0 without any error that 1 / sqrt(eps)
would enlarge.  Widths of every form whose reciprocal, rounded, times their own multiple is not the multiplicand."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402
from layer_util import TYPES  # noqa: E402

VALUES = [1.0, -3.0, 5.0, 7.0, 19.0, 52.0, 100.0, 120.0, -248.0]     # in every type
# one wave (whole vectors, with a tail, fewer than one), 4 waves, 16 waves, rows that are not held
WIDTHS = [7, 41, 120, 488, 953, 1952, 3995, 4067, 7808, 15_616, 16_247, 20_520, 20_655]


def config(rows, dim, kind):
    code = E.ea_type(kind)
    return E.LayerNorm(rows=rows, dim=dim, x_stride=dim, y_stride=dim, eps=1e-5, x_type=code, y_type=code, w_type=E.EA_F32)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("dim", WIDTHS)
def test_rows_of_one_value_give_the_bias(dim, kind):
    """Sums of at most 248 x 20,655 are exact in binary32 in any order."""
    dtype, rows = TYPES[kind], len(VALUES)
    values = torch.tensor(VALUES, device="cuda")
    x = values[:, None].expand(rows, dim).to(dtype).contiguous()
    gen = torch.Generator(device="cuda").manual_seed(dim)
    w, b = torch.randn(dim, device="cuda", generator=gen) * 50, torch.randn(dim, device="cuda", generator=gen)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    E.ea_layer_norm(config(rows, dim, dtype), x, w, b, y, mean, rstd)
    assert torch.equal(mean, values)
    assert torch.equal(y, b.to(dtype).expand(rows, dim))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("dim", WIDTHS)
def test_gradients_along_the_mean_and_the_row_vanish(dim, kind):
    """For x of 1 and -1 in pairs (0 at an odd end), a mean of 0 and rstd of 1: a gradient of one value c has the mean c, and
    its sum with x is 0; one of c x has the mean 0, and c as its mean product with x (of an even width).  dx is what is
    left of them, 0, so that with `add` it is `add`."""
    dtype = TYPES[kind]
    sign = torch.where(torch.arange(dim, device="cuda") % 2 == 0, 1.0, -1.0)
    if dim % 2:
        sign[-1] = 0
    along = [torch.ones_like(sign)] + ([sign] if dim % 2 == 0 else [])
    dy = torch.stack([c * v for v in along for c in VALUES]).to(dtype)
    rows = len(dy)
    x = sign.expand(rows, dim).to(dtype).contiguous()
    mean, rstd = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    add = torch.randn((rows, dim), device="cuda", generator=torch.Generator(device="cuda").manual_seed(dim)).to(dtype)
    for a in (None, add):
        dx = torch.empty_like(x)
        E.ea_layer_norm_grad(config(rows, dim, dtype), x, dy, None, mean, rstd, a, dx, None, None, False, None)
        assert bool((dx == (0 if a is None else a)).all())


@pytest.mark.parametrize("dim", [41, 488, 953, 1952, 16_247, 20_655])
def test_infinite_sums_have_infinite_means(dim):
    """A row's mean is its sum's quotient where that is an infinity too; the gradient of a row whose dy holds one is what the
    formula's operations give: -infinity where nothing else is infinite."""
    inf = float("inf")
    x = torch.ones((4, dim), device="cuda")
    x[0, 5], x[1, dim - 1], x[2, 0], x[2, 1] = inf, -inf, inf, -inf
    x[3, :2] = 3e38
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    c = config(4, dim, torch.float32)
    E.ea_layer_norm(c, x, None, None, y, mean, rstd)
    assert mean[0].item() == inf and mean[1].item() == -inf and mean[2].isnan() and mean[3].item() == inf
    assert bool(y.isnan().all())
    # x of 0 with a mean of 0: dx = rstd (dy - mean(dy)), and the mean is infinite
    dy, dx = torch.ones_like(x), torch.empty_like(x)
    dy[1, :2] = 3e38
    E.ea_layer_norm_grad(c, torch.zeros_like(x), dy, None, torch.zeros_like(mean), torch.ones_like(rstd), None, dx, None, None,
                         False, None)
    assert bool((dx[1] == -inf).all()) and bool(dx[::2].isfinite().all())
