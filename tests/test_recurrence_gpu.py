"""The gated linear recurrence and its gradient against 64 bits, step by step: lengths from 0 and 1 to several tiles
and segments, types, odd widths, row gaps, padded sequences, states carried over, in place, gates of 0 and 1 and past
the tables' ends, NaN behind a sequence's end, other streams, graphs."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402
import paper_2205_14473_amd as E  # noqa: E402
import train_util as R  # noqa: E402
from layer_util import TYPES  # noqa: E402

PLAIN, SIGMOID = 0, 1


def config(b, n, dim, x, g, gate, gap=(0, 0, 0)):
    return E.Recurrence(batch=b, length=n, dim=dim, x_stride=dim + gap[0], g_stride=dim + gap[1], y_stride=dim + gap[2],
                        gate=gate, x_type=E.ea_type(x), g_type=E.ea_type(g))


def inputs(b, n, dim, x, g, gate, seed=0):
    gen = torch.Generator().manual_seed(seed + b * 1_000_003 + n * 101 + dim)
    gv = torch.randn((b, n, dim), generator=gen) * 1.5 + torch.rand(dim, generator=gen) * 5
    gv = (torch.tanh(gv * 0.5) if gate == PLAIN else gv).to(g)
    xv, dy = torch.randn((b, n, dim), generator=gen).to(x), torch.randn((b, n, dim), generator=gen).to(x)
    h0, dh = (torch.randn((b, dim), generator=gen) for _ in range(2))
    return gv, xv, h0, dy, dh


def device_rows(v, stride, dtype, shift):
    """(allocation, [b, n, dim] of it) with gaps between rows."""
    b, n, dim = v if isinstance(v, tuple) else v.shape
    flat, view = L.spaced((b * n, dim), stride, dtype, shift)
    out = torch.as_strided(flat, (b, n, dim), (n * stride, stride, 1), shift)
    if not isinstance(v, tuple):
        out.copy_(v)
    return flat, view, out


class Run:
    """Forward and gradient of one case, and the checks of both."""

    def __init__(self, b, n, dim, x, g, gate, gap=(0, 0, 0), shift=0, lengths=None, start=True, seed=0, values=None):
        self.c = c = config(b, n, dim, x, g, gate, gap)
        gv, xv, h0, dy, dh = values or inputs(b, n, dim, x, g, gate, seed)
        if not start:
            h0, dh = torch.zeros_like(h0), torch.zeros_like(dh)
        self.counts = torch.full((b,), n) if lengths is None else torch.tensor(lengths).clamp(0, n)
        ld = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
        if lengths is not None:                     # what lies behind an end is not read
            past = torch.arange(n)[None, :, None] >= self.counts[:, None, None]
            gq, xq, dq = (torch.where(past, torch.full((), float("nan"), dtype=v.dtype), v) for v in (gv, xv, dy))
        else:
            gq, xq, dq = gv, xv, dy
        gd, xd = device_rows(gq, c.g_stride, g, shift)[2], device_rows(xq, c.x_stride, x, shift)[2]
        dyd = device_rows(dq, c.y_stride, x, shift)[2]
        yf, yv, y = device_rows((b, n, dim), c.y_stride, x, shift)
        blocks = -(-n // 64)
        assert E.ea_recurrence_states_bytes(c) == 4 * b * blocks * dim
        states = torch.full((b * blocks * dim + 4,), L.GUARD, device="cuda")
        last = torch.full((b * dim + 4,), L.GUARD, device="cuda")
        need = E.ea_recurrence_workspace_bytes(c)
        wsf = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
        ws = wsf[:need] if need else None
        h0d, dhd = (h0.cuda(), dh.cuda()) if start else (None, None)
        E.ea_recurrence(c, gd, xd, h0d, ld, y, states[:-4], last[:-4], ws)
        torch.cuda.synchronize()
        assert bool((wsf[need:] == 0xA5).all()) and bool((states[-4:] == L.GUARD).all()) and bool((last[-4:] == L.GUARD).all())
        assert L.guards_kept(yf, yv, shift)
        want = L.Recurrence(gv.double(), xv.double(), h0.double(), self.counts, gate)
        self.y, self.states, self.last = y, states[:-4].view(b, blocks, dim), last[:-4].view(b, dim)
        R.within(y, want.y, want.bound + L.rounding(want.y, x), "y")
        R.within(self.states, want.states, want.states_bound, "states")
        R.within(self.last, want.h_last, want.h_last_bound, "h_last")
        # without states and last: the same
        y2 = torch.empty_like(y.contiguous()) if gap[2] == 0 else device_rows((b, n, dim), c.y_stride, x, shift)[2]
        E.ea_recurrence(c, gd, xd, h0d, ld, y2, None, None, ws)
        assert torch.equal(y, y2)
        df, dv, dx = device_rows((b, n, dim), c.x_stride, x, shift)
        gf, gv2, dg = device_rows((b, n, dim), c.g_stride, g, shift)
        dh0 = torch.full((b * dim + 4,), L.GUARD, device="cuda")
        E.ea_recurrence_grad(c, gd, xd, want.states.float().cuda(), ld, dyd, dhd, dg, dx, dh0[:-4], ws)
        torch.cuda.synchronize()
        assert bool((wsf[need:] == 0xA5).all()) and bool((dh0[-4:] == L.GUARD).all())
        assert L.guards_kept(df, dv, shift) and L.guards_kept(gf, gv2, shift)
        back = L.RecurrenceGrad(gv.double(), xv.double(), h0.double(), self.counts, gate, dy.double(), dh.double())
        self.dx, self.dg, self.dh0 = dx, dg, dh0[:-4].view(b, dim)
        R.within(dx, back.dx, back.dx_bound + L.rounding(back.dx, x), "dx")
        # the states given are the true ones, rounded: within the forward's bound of them
        R.within(dg, back.dg, back.dg_bound + L.rounding(back.dg, g), "dg")
        R.within(self.dh0, back.dh0, back.dh0_bound, "dh0")


LENGTHS = [1, 2, 7, 8, 9, 15, 16, 17, 33, 63, 64, 65, 100, 127, 128, 129, 191, 192, 193, 256, 300]


@pytest.mark.parametrize("gate", [PLAIN, SIGMOID])
@pytest.mark.parametrize("n", LENGTHS)
def test_lengths(n, gate):
    Run(3, n, 70, torch.float32, torch.float32, gate)


@pytest.mark.parametrize("gate", [PLAIN, SIGMOID])
@pytest.mark.parametrize("dim", [1, 2, 3, 63, 64, 65, 127, 128, 129, 257, 768])
def test_widths(dim, gate):
    gap, shift = ((0, 0, 0), 0) if dim % 2 == 0 else ((3, 1, 5), 1)
    Run(2, 37, dim, torch.bfloat16, torch.bfloat16, gate, gap, shift)
    Run(1, 140, dim, torch.bfloat16, torch.float32, gate, gap, shift, start=False)


@pytest.mark.parametrize("gate", [PLAIN, SIGMOID])
@pytest.mark.parametrize("x", TYPES)
@pytest.mark.parametrize("g", TYPES)
def test_types(x, g, gate):
    Run(2, 150, 131, TYPES[x], TYPES[g], gate, (1, 2, 3), 1)


@pytest.mark.parametrize("gate", [PLAIN, SIGMOID])
@pytest.mark.parametrize("b,n,dim", [(1, 513, 64), (1, 640, 65), (1, 1025, 130), (2, 2047, 40), (1, 4100, 16), (3, 700, 300)])
def test_segments(b, n, dim, gate):
    assert E.ea_recurrence_workspace_bytes(config(b, n, dim, torch.float32, torch.float32, gate)) > 0
    Run(b, n, dim, torch.float32, torch.float32, gate)
    Run(b, n, dim, torch.bfloat16, torch.bfloat16, gate, start=False)


@pytest.mark.parametrize("gate", [PLAIN, SIGMOID])
@pytest.mark.parametrize("n,lengths", [(1, [0, 1, 1]), (8, [0, 8, 3, 7]), (70, [64, 0, 70, 1, 65, 63]), (200, [129, 0, 200, 128, 1, 64]),
                                       (150, [-5, 1000, 2 ** 31 - 1, -2 ** 31]), (1500, [1, 0, 1500, 640, 641, 1025])])
def test_padded_sequences(n, lengths, gate):
    r = Run(len(lengths), n, 66, torch.float32, torch.bfloat16, gate, (0, 4, 2), lengths=lengths)
    past = torch.arange(n)[None, :] >= r.counts[:, None]
    for v in (r.y, r.dx, r.dg):
        assert bool((v.cpu()[past] == 0).all())


@pytest.mark.parametrize("n", [1, 9, 130, 600])
def test_state_carried_over(n):
    """A sequence in two calls, the state of the first one carried in place."""
    b, dim = 2, 96
    gv, xv, h0, _, _ = inputs(b, 2 * n, dim, torch.float32, torch.float32, SIGMOID)
    want = L.Recurrence(gv.double(), xv.double(), h0.double(), torch.full((b,), 2 * n), SIGMOID)
    h = h0.cuda()
    for part in (slice(0, n), slice(n, 2 * n)):
        c = config(b, n, dim, torch.float32, torch.float32, SIGMOID)
        need = E.ea_recurrence_workspace_bytes(c)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        y = torch.empty((b, n, dim), device="cuda")
        E.ea_recurrence(c, gv[:, part].contiguous().cuda(), xv[:, part].contiguous().cuda(), h, None, y, None, h, ws)
        R.within(y, want.y[:, part], want.bound[:, part], "y")
    R.within(h, want.h_last, want.h_last_bound, "h_last")


@pytest.mark.parametrize("n", [5, 700])
def test_ends_in_place(n):
    b, dim = 2, 70
    c = config(b, n, dim, torch.float32, torch.float32, SIGMOID)
    gv, xv, h0, dy, dh = (v.cuda() for v in inputs(b, n, dim, torch.float32, torch.float32, SIGMOID))
    need = E.ea_recurrence_workspace_bytes(c)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    y, dg, dx = (torch.empty_like(xv) for _ in range(3))
    states = torch.empty((b, -(-n // 64), dim), device="cuda")
    last, first = torch.empty_like(h0), torch.empty_like(h0)
    E.ea_recurrence(c, gv, xv, h0, None, y, states, last, ws)
    E.ea_recurrence_grad(c, gv, xv, states, None, dy, dh, dg, dx, first, ws)
    E.ea_recurrence(c, gv, xv, h0, None, y, states, h0, ws)
    E.ea_recurrence_grad(c, gv, xv, states, None, dy, dh, dg, dx, dh, ws)
    assert torch.equal(h0, last) and torch.equal(dh, first)


@pytest.mark.parametrize("n", [3, 200, 900])
def test_gates_at_their_ends(n):
    """Plain gates of 0, 1 and -1 and sigmoids that round to 0 and 1 (a gate of 1 keeps the state, one of 0 drops it)."""
    b, dim = 2, 72
    gv, xv, h0, dy, dh = inputs(b, n, dim, torch.float32, torch.float32, PLAIN)
    pick = torch.randint(0, 4, gv.shape, generator=torch.Generator().manual_seed(n))
    plain = torch.tensor([0.0, 1.0, -1.0, 0.5])[pick]
    Run(b, n, dim, torch.float32, torch.float32, PLAIN, values=(plain, xv, h0, dy, dh))
    logits = torch.tensor([-200.0, 200.0, float("inf"), 1.0])[pick]
    logits[:, :, ::5] = -float("inf")
    run = (logits, xv, h0, dy, dh)
    c = config(b, n, dim, torch.float32, torch.float32, SIGMOID)
    need = E.ea_recurrence_workspace_bytes(c)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    y, dg, dx = (torch.empty((b, n, dim), device="cuda") for _ in range(3))
    states, dh0 = torch.empty((b, -(-n // 64), dim), device="cuda"), torch.empty((b, dim), device="cuda")
    gd, xd, hd, dyd, dhd = (v.cuda() for v in run)
    E.ea_recurrence(c, gd, xd, hd, None, y, states, None, ws)
    E.ea_recurrence_grad(c, gd, xd, states, None, dyd, dhd, dg, dx, dh0, ws)
    cut = logits.clamp(-100, 100).double()
    want = L.RecurrenceGrad(cut, xv.double(), h0.double(), torch.full((b,), n), SIGMOID, dy.double(), dh.double())
    f = L.Recurrence(cut, xv.double(), h0.double(), torch.full((b,), n), SIGMOID)
    R.within(y, f.y, f.bound + 2.0 ** -120, "y")
    R.within(dx, want.dx, want.dx_bound + 2.0 ** -120, "dx")
    R.within(dg, want.dg, want.dg_bound + 2.0 ** -120, "dg")


@pytest.mark.parametrize("dim,n,lengths", [(70, 70_001, [70_001, 66_000]), (3, 140_000, [131_073, 140_000, 1]), (130, 33_000, [33_000])])
def test_long_sequences_in_whole_numbers(dim, n, lengths):
    """Gates of 1, -1 and now and then 0 over small whole numbers: every sum is exact in binary32, in any order, and the
    results are equal to those of the steps.  Long enough for chunks, groups and several stretches of them."""
    rng = np.random.default_rng(n)
    b = len(lengths)
    a = rng.choice([1, 1, 1, -1], (b, n, dim)) * (rng.random((b, n, dim)) > 0.002)
    x, dy = rng.integers(-2, 3, (b, n, dim)), rng.integers(-2, 3, (b, n, dim))
    h0, dh = rng.integers(-9, 10, (b, dim)), rng.integers(-9, 10, (b, dim))
    y, before, dx, dg = (np.zeros((b, n, dim), np.int64) for _ in range(4))
    last, first = h0.copy(), dh.copy()
    for i, steps in enumerate(lengths):
        h = h0[i]
        for t in range(steps):
            before[i, t] = h
            h = a[i, t] * h + x[i, t]
            y[i, t] = h
        last[i], e = h, dh[i]
        for t in range(steps - 1, -1, -1):
            d = dy[i, t] + e
            dx[i, t], dg[i, t] = d, d * before[i, t]
            e = a[i, t] * d
        first[i] = e
    assert max(abs(v).max() for v in (y, dx, dg)) < 1 << 24
    c = config(b, n, dim, torch.float32, torch.float32, PLAIN)
    ws = torch.empty(E.ea_recurrence_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    dev = lambda v: torch.from_numpy(v).float().cuda()  # noqa: E731
    gd, xd, got = dev(a), dev(x), torch.empty((b, n, dim), device="cuda")
    ld = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    states, hl = torch.empty((b, -(-n // 64), dim), device="cuda"), torch.empty((b, dim), device="cuda")
    E.ea_recurrence(c, gd, xd, dev(h0), ld, got, states, hl, ws)
    assert torch.equal(got.cpu().long(), torch.from_numpy(y)) and torch.equal(hl.cpu().long(), torch.from_numpy(last))
    gx, gg = torch.empty_like(got), torch.empty_like(got)
    E.ea_recurrence_grad(c, gd, xd, states, ld, dev(dy), dev(dh), gg, gx, hl, ws)
    assert torch.equal(gx.cpu().long(), torch.from_numpy(dx)) and torch.equal(gg.cpu().long(), torch.from_numpy(dg))
    assert torch.equal(hl.cpu().long(), torch.from_numpy(first))


def test_growing_gates_from_zero_states_stay_what_the_steps_give():
    """Gates of 2^20 multiply to infinity within a tile; a state of 0 under inputs of 0 stays 0."""
    n, dim = 300, 64
    g, x = torch.full((1, n, dim), 2.0 ** 20, device="cuda"), torch.zeros((1, n, dim), device="cuda")
    c = config(1, n, dim, torch.float32, torch.float32, PLAIN)
    y, last = torch.full((1, n, dim), 3.0, device="cuda"), torch.empty((1, dim), device="cuda")
    ws = torch.empty(max(1, E.ea_recurrence_workspace_bytes(c)), dtype=torch.uint8, device="cuda")
    E.ea_recurrence(c, g, x, None, None, y, None, last, ws)
    assert bool((y == 0).all()) and bool((last == 0).all())


def test_nan_stays_in_its_channel_and_after_its_step():
    b, n, dim = 2, 700, 130
    gv, xv, h0, dy, dh = inputs(b, n, dim, torch.float32, torch.float32, SIGMOID)
    c = config(b, n, dim, torch.float32, torch.float32, SIGMOID)
    ws = torch.empty(E.ea_recurrence_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    out = []
    for bad in (False, True):
        x = xv.clone()
        if bad:
            x[0, 333, 7] = float("nan")
        y = torch.empty((b, n, dim), device="cuda")
        E.ea_recurrence(c, gv.cuda(), x.cuda(), h0.cuda(), None, y, None, None, ws)
        out.append(y.cpu())
    hit = torch.zeros((b, n, dim), dtype=torch.bool)
    hit[0, 333:, 7] = True
    assert torch.equal(out[0][~hit], out[1][~hit]) and bool(out[1][hit].isnan().all())


@pytest.mark.parametrize("b,n", [(0, 5), (3, 0), (0, 0)])
def test_nothing_to_do(b, n):
    c = config(b, n, 10, torch.float32, torch.float32, SIGMOID)
    assert E.ea_recurrence_workspace_bytes(c) == 0 and E.ea_recurrence_states_bytes(c) == 0
    none, st = torch.empty((b, n, 10), device="cuda"), torch.empty((b, 0, 10), device="cuda")
    h0, last = torch.randn((b, 10), device="cuda"), torch.full((b, 10), 9.0, device="cuda")
    E.ea_recurrence(c, none, none, h0, None, none, st, last, None)
    assert torch.equal(last, h0)
    E.ea_recurrence(c, none, none, None, None, none, None, last, None)
    assert bool((last == 0).all())
    E.ea_recurrence_grad(c, none, none, st, None, none, h0, none, none, last, None)
    assert torch.equal(last, h0)


@pytest.mark.parametrize("gate", [PLAIN, SIGMOID])
def test_gradient_by_differences(gate):
    """Along random directions of g, x and h0, by the 64-bit steps: central differences of a step of 2^-12."""
    b, n, dim = 2, 90, 20
    v = inputs(b, n, dim, torch.float32, torch.float32, gate, seed=4)
    r = Run(b, n, dim, torch.float32, torch.float32, gate, values=v, lengths=[90, 71])
    gv, xv, h0, dy, dh = (t.double() for t in v)
    on = (torch.arange(n)[None, :] < r.counts[:, None])[..., None]

    def f(g, x, h):
        w = L.Recurrence(g, x, h, r.counts, gate)
        return ((w.y * dy * on).sum() + (w.h_last * dh).sum()).item()

    at, h = [gv, xv, h0], 2.0 ** -12
    for k, got in enumerate((r.dg, r.dx, r.dh0)):
        D = torch.randn(at[k].shape, dtype=torch.float64, generator=torch.Generator().manual_seed(k))
        side = [f(*[t + s * h * D if i == k else t for i, t in enumerate(at)]) for s in (1, -1)]
        slope, terms = (side[0] - side[1]) / (2 * h), got.cpu().double() * D
        # h^2 / 6 of a third derivative, of the terms' size over the gates' few hundred products
        assert abs(slope - terms.sum().item()) <= 1e-5 * terms.abs().sum().item() + 1e-4


def test_graph_streams_and_the_same_bits():
    for b, n, dim in ((5, 300, 200), (1, 3000, 130)):
        gv, xv, h0, dy, dh = (t.cuda() for t in inputs(b, n, dim, torch.bfloat16, torch.bfloat16, SIGMOID))
        c = config(b, n, dim, torch.bfloat16, torch.bfloat16, SIGMOID)
        need = E.ea_recurrence_workspace_bytes(c)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
        outs = [torch.zeros_like(xv) for _ in range(3)]
        states, last, first = torch.zeros((b, -(-n // 64), dim), device="cuda"), torch.zeros_like(h0), torch.zeros_like(h0)

        def both(stream=None):
            E.ea_recurrence(c, gv, xv, h0, None, outs[0], states, last, ws, stream=stream)
            E.ea_recurrence_grad(c, gv, xv, states, None, dy, dh, outs[1], outs[2], first, ws, stream=stream)

        every = lambda: [t.clone() for t in outs + [states, last, first]]  # noqa: E731
        both()
        torch.cuda.synchronize()
        held, s = every(), torch.cuda.Stream()
        both(s)
        s.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, every()))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            both()
        for k in range(3):
            xv.mul_(1.5)
            graph.replay()
            torch.cuda.synchronize()
            got = every()
            both()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, every()))


def test_rows_past_32_bit_offsets():
    n, dim, stride = 40, 6, 1 << 27
    flat = torch.zeros(n * stride, dtype=torch.bfloat16, device="cuda")
    gv, xv, h0, _, _ = inputs(1, n, dim, torch.bfloat16, torch.bfloat16, SIGMOID)
    x = torch.as_strided(flat, (1, n, dim), (n * stride, stride, 1))
    y = torch.as_strided(flat, (1, n, dim), (n * stride, stride, 1), 64)
    x.copy_(xv)
    c = E.Recurrence(batch=1, length=n, dim=dim, x_stride=stride, g_stride=dim, y_stride=stride, gate=SIGMOID,
                     x_type=E.EA_BF16, g_type=E.EA_BF16)
    E.ea_recurrence(c, gv.cuda(), x, h0.cuda(), None, y, None, None, None)
    want = L.Recurrence(gv.double(), xv.double(), h0.double(), torch.full((1,), n), SIGMOID)
    R.within(y, want.y, want.bound + L.rounding(want.y, torch.bfloat16), "y")
