"""The recurrence near the ends of binary32's range: gates whose products over a wave's steps come near it and stay inside,
infinite inputs, products that fall to 0."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402

PLAIN, SIGMOID = 0, 1


def run(g, x, h0, gate):
    b, n, dim = x.shape
    c = E.Recurrence(batch=b, length=n, dim=dim, x_stride=dim, g_stride=dim, y_stride=dim, gate=gate, x_type=E.EA_F32,
                     g_type=E.EA_F32)
    ws = torch.empty(max(16, E.ea_recurrence_workspace_bytes(c)), dtype=torch.uint8, device="cuda")
    y, states = torch.empty_like(x), torch.empty((b, -(-n // 64), dim), device="cuda")
    last = torch.empty((b, dim), device="cuda")
    E.ea_recurrence(c, g, x, h0, None, y, states, last, ws)
    return c, ws, y, states, last


@pytest.mark.parametrize("n", [10, 16, 100, 300, 5000, 70_000])
def test_growing_and_shrinking_gates(n):
    """16 gates of 2^7, then 16 of 2^-7: the state moves between 1 and 2^112, every product of some of the steps lies within
    2^-112 and 2^112, and all are powers of two: exact in any order, forward and back."""
    dim = 65
    power = torch.where(torch.arange(n) % 32 < 16, 7, -7)
    at = power.cumsum(0)                                # the exponent behind each step
    sign = torch.where(torch.arange(dim) % 2 == 0, 1.0, -1.0).double()
    g = (2.0 ** power.double())[None, :, None].expand(1, n, dim).float().contiguous().cuda()
    x, h0 = torch.zeros((1, n, dim), device="cuda"), sign[None].float().cuda()
    c, ws, y, states, last = run(g, x, h0, PLAIN)
    want = (2.0 ** at.double())[:, None] * sign
    assert torch.equal(y[0].cpu().double(), want)
    assert torch.equal(last[0].cpu().double(), want[-1])
    before = torch.cat([torch.zeros(1, dtype=at.dtype), at[:-1]])
    assert torch.equal(states[0].cpu().double(), (2.0 ** before[::64].double())[:, None] * sign)
    # d_t is the product of the gates behind step t, times dh_last
    dg, dx, dh0 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
    E.ea_recurrence_grad(c, g, x, states, None, x, torch.ones_like(h0), dg, dx, dh0, ws)
    d = 2.0 ** (at[-1] - at).double()
    assert torch.equal(dx[0].cpu().double(), d[:, None].expand(n, dim))
    assert torch.equal(dg[0].cpu().double(), (d * 2.0 ** before.double())[:, None] * sign)
    assert torch.equal(dh0[0].cpu().double(), torch.full((dim,), 2.0 ** int(at[-1]), dtype=torch.float64))


@pytest.mark.parametrize("gate", [PLAIN, SIGMOID])
@pytest.mark.parametrize("n", [40, 300, 3000])
def test_products_that_fall_to_0_and_infinities(n, gate):
    """Gates of a half: from 150 steps on nothing of the state is left, none of it NaN; an infinite input is infinite where it
    arrives, and no later state of its channel is finite."""
    dim, at = 66, 20
    g = torch.full((1, n, dim), 0.5 if gate == PLAIN else 0.0, device="cuda")
    x = torch.zeros((1, n, dim), device="cuda")
    h0 = torch.full((1, dim), 2.0 ** 100, device="cuda")
    y = run(g, x, h0, gate)[2]
    exact = 2.0 ** (99 - torch.arange(n, dtype=torch.float64))
    whole = exact >= 2.0 ** -126                       # smaller ones may be rounded, or be 0 already
    assert torch.equal(y[0, whole.cuda()].cpu().double(), exact[whole][:, None].expand(-1, dim))
    assert bool((y[0, ~whole.cuda()].abs() <= 2.0 ** -126).all())
    x[0, at, 5] = float("inf")
    z = run(g, x, h0, gate)[2]
    assert bool((z[0, at:at + 12, 5] == float("inf")).all()) and not z[0, at:, 5].isfinite().any()
    z[0, :, 5] = y[0, :, 5]
    assert torch.equal(y, z)
