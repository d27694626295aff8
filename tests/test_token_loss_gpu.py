"""The token loss and its gradient against 64 bits: vocabularies of every form, types, row gaps, misaligned rows, targets
that do not count, masked logits, infinities and NaN, mean and sum, in place, many rows, other streams, graphs."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402
import paper_2205_14473_amd as E  # noqa: E402
import train_util as R  # noqa: E402
from layer_util import TYPES, U32  # noqa: E402


def config(rows, vocab, kind, bits=64, gap=0, dgap=0, scale=1.0, mean=True):
    return E.TokenLoss(rows=rows, vocab=vocab, logits_stride=vocab + gap, dlogits_stride=vocab + dgap, scale=scale,
                       type=E.ea_type(kind), index_bits=bits, reduction=E.EA_REDUCE_MEAN if mean else E.EA_REDUCE_SUM)


def inputs(rows, vocab, kind, seed=0):
    gen = torch.Generator().manual_seed(seed + rows * 31 + vocab)
    z = torch.randn((rows, vocab), generator=gen) * 3
    t = torch.randint(0, vocab, (rows,), generator=gen)
    z[torch.arange(rows), t] += 4
    if rows > 2:
        t[::3] = torch.tensor([-100, vocab, -1, 2 ** 31 - 1, -2 ** 31]).repeat(rows)[:len(t[::3])]
    return z.to(kind), t


def run(z, t, c, grad=True, shift=0, in_place=False):
    """(loss, total, count, dlogits), everything around them checked."""
    rows, vocab = z.shape
    _, zd = L.spaced(z, c.logits_stride, z.dtype, shift)
    flat, dz = L.spaced((rows, vocab), c.dlogits_stride, z.dtype, shift)
    loss, total = torch.full((rows + 2,), L.GUARD, device="cuda"), torch.full((3,), L.GUARD, device="cuda")
    count = torch.full((3,), 55, dtype=torch.int32, device="cuda")
    need = E.ea_token_loss_workspace_bytes(c)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    td = t.to(torch.int32 if c.index_bits == 32 else torch.int64).cuda()
    E.ea_token_loss(c, zd, td, loss[1:-1], total[1:2], count[1:2], (zd if in_place else dz) if grad else None,
                    ws[:need] if need else None)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xA5).all()), "a write past the workspace"
    assert L.guards_kept(flat, dz if grad and not in_place else dz[:0], shift)
    for v in (loss, total, count):
        assert v[0].item() == 55 and v[-1].item() == 55
    return loss[1:-1], total[1], count[1], zd if in_place else dz


def check(got, z, t, c, grad=True):
    want = L.Loss(z.double(), t, c.scale, c.reduction == E.EA_REDUCE_MEAN)
    R.within(got[0], want.loss, want.loss_bound, "loss")
    assert abs(got[1].item() - want.total) <= want.total_bound
    assert got[2].item() == want.count
    if grad:
        R.within(got[3], want.dz, want.dz_bound + L.rounding(want.dz, z.dtype), "dlogits")


VOCABS = [1, 2, 3, 7, 8, 9, 255, 511, 512, 513, 1000, 1024, 1025, 2047, 2049, 4096, 4097, 8191, 8193, 16_385, 30_001, 50_257,
          65_537, 70_000, 131_073, 140_001]


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_vocabularies(vocab, kind):
    rows = 7 if vocab < 5000 else 4
    z, t = inputs(rows, vocab, TYPES[kind])
    gap, dgap, shift = (0, 0, 0) if vocab % 2 == 0 else (3, 1, 1)
    scale = 1000.0 if kind == "f16" else 0.7
    c = config(rows, vocab, TYPES[kind], 32 if vocab % 3 == 0 else 64, gap, dgap, scale, mean=vocab % 4 != 0)
    got = run(z, t, c, shift=shift)
    check(got, z, t, c)
    alone = run(z, t, c, grad=False, shift=shift)
    assert all(torch.equal(a, b) for a, b in zip(got[:3], alone[:3]))


@pytest.mark.parametrize("mean", [True, False])
@pytest.mark.parametrize("rows,vocab", [(1, 50), (2, 3000), (5, 20), (1023, 5), (4096, 3), (4097, 3), (9000, 17), (3000, 600), (2100, 1500),
                                        (70_000, 2)])
def test_rows(rows, vocab, mean):
    z, t = inputs(rows, vocab, torch.float32)
    c = config(rows, vocab, torch.float32, mean=mean, scale=3.0)
    check(run(z, t, c), z, t, c)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [100, 5000, 50_257, 140_001])
def test_in_place(vocab, kind):
    z, t = inputs(5, vocab, TYPES[kind])
    c = config(5, vocab, TYPES[kind], scale=500.0)
    a, b = run(z, t, c), run(z, t, c, in_place=True)
    assert all(torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("vocab", [40, 1500, 20_000, 70_000])
def test_masked_logits(vocab):
    """Logits of -infinity and of the type's lowest value, the largest logits of all, a row with one left."""
    z, t = inputs(6, vocab, torch.float32)
    low = torch.finfo(torch.float32).min
    z[1, ::2], z[2, 1::2] = -float("inf"), low
    t[:] = torch.tensor([0, 1, 0, 3, 5, 7])
    z[3] = -float("inf")
    z[3, 3] = -2.5
    z[4] = low
    z[4, 5] = 3e38
    c = config(6, vocab, torch.float32, mean=False)
    loss, total, count, dz = run(z, t, c)
    zw = torch.where(z < -1e38, torch.full((), -1e4), z)
    zw[4] = -1e4
    zw[4, 5] = 0.0
    want = L.Loss(zw.double(), t, 1.0, False)
    R.within(loss, want.loss, want.loss_bound, "loss")
    R.within(dz, want.dz, want.dz_bound, "dlogits")
    assert loss[3].item() == 0.0 and bool((dz[3] == 0).all()) and count.item() == 6
    assert bool((dz[1, ::2] == 0).all()) and bool((dz[2, 1::2] == 0).all())
    t[1] = 0                                        # a target that is masked: an infinite loss, a gradient of -1 there
    loss, total, _, dz = run(z, t, c)
    assert loss[1].item() == float("inf") and total.item() == float("inf") and dz[1, 0].item() == -1.0


@pytest.mark.parametrize("vocab", [40, 1500, 20_000, 70_000])
def test_infinities_and_nan_stay_in_rows_that_count(vocab):
    z, t = inputs(9, vocab, torch.float32)
    t[:] = torch.arange(9)
    good = config(9, vocab, torch.float32, mean=False)
    a = run(z, t, good)
    z[1], z[3, vocab - 1], z[5, 0] = -float("inf"), float("nan"), float("inf")
    z[7] = float("nan")
    t[7] = -100                                     # not read
    b = run(z, t, good)
    same = [0, 2, 4, 6, 8]
    assert torch.equal(a[0][same], b[0][same]) and torch.equal(a[3][same], b[3][same])
    for k in (1, 3, 5):
        assert b[0][k].isnan() and b[3][k].isnan().all()
    assert b[0][7].item() == 0 and bool((b[3][7] == 0).all()) and b[1].isnan() and b[2].item() == 8


@pytest.mark.parametrize("mean", [True, False])
def test_nothing_counts(mean):
    c = config(5, 30, torch.float32, mean=mean)
    z, _ = inputs(5, 30, torch.float32)
    loss, total, count, dz = run(z, torch.full((5,), -100), c)
    assert total.item() == 0 and count.item() == 0 and bool((loss == 0).all()) and bool((dz == 0).all())
    c = config(0, 30, torch.float32, mean=mean)
    assert E.ea_token_loss_workspace_bytes(c) == 0
    loss, total, count, dz = run(z[:0], torch.empty(0, dtype=torch.int64), c)
    assert total.item() == 0 and count.item() == 0


def test_optional_outputs():
    z, t = inputs(6, 77, torch.bfloat16)
    c = config(6, 77, torch.bfloat16)
    want = run(z, t, c)
    total, ws = torch.empty(1, device="cuda"), torch.empty(E.ea_token_loss_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    E.ea_token_loss(c, z.cuda(), t.cuda(), None, total, None, None, ws)
    assert total.item() == want[1].item()


def test_gradient_by_differences():
    """Along a random direction of the logits, by the 64-bit loss: central differences of a step of 2^-12."""
    z, t = inputs(8, 120, torch.float32)
    c = config(8, 120, torch.float32, scale=1.0)
    dz = run(z, t, c)[3].cpu().double()
    D = torch.randn(z.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(2))
    h = 2.0 ** -12
    side = [L.Loss(z.double() + s * h * D, t, 1.0, True).total for s in (1, -1)]
    assert abs((side[0] - side[1]) / (2 * h) - (dz * D).sum().item()) <= 1e-5 * (dz * D).abs().sum().item() + 1e-6


def test_rows_past_32_bit_offsets():
    vocab, stride = 50, (1 << 31) + 6
    flat = torch.zeros(stride + 2 * vocab, dtype=torch.bfloat16, device="cuda")
    z, _ = inputs(2, vocab, torch.bfloat16)
    t = torch.tensor([3, 4])
    zd = torch.as_strided(flat, (2, vocab), (stride, 1))
    zd.copy_(z)
    c = E.TokenLoss(rows=2, vocab=vocab, logits_stride=stride, dlogits_stride=stride, scale=1.0, type=E.EA_BF16, index_bits=64)
    ws = torch.empty(E.ea_token_loss_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    total = torch.empty(1, device="cuda")
    E.ea_token_loss(c, zd, t.cuda(), None, total, None, zd, ws)
    want = L.Loss(z.double(), t, 1.0, True)
    assert abs(total.item() - want.total) <= want.total_bound
    R.within(zd, want.dz, want.dz_bound + L.rounding(want.dz, torch.bfloat16), "dlogits")


def test_graph_streams_and_the_same_bits():
    for rows, vocab in ((700, 900), (5000, 300), (40, 50_257)):
        z, t = inputs(rows, vocab, torch.bfloat16)
        c = config(rows, vocab, torch.bfloat16, scale=100.0)
        zd, td = z.cuda(), t.cuda()
        ws = torch.empty(E.ea_token_loss_workspace_bytes(c), dtype=torch.uint8, device="cuda")
        loss, total, count = torch.zeros(rows, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        dz = torch.zeros_like(zd)

        def call(stream=None):
            E.ea_token_loss(c, zd, td, loss, total, count, dz, ws, stream=stream)

        every = lambda: [v.clone() for v in (loss, total, count, dz)]  # noqa: E731
        call()
        torch.cuda.synchronize()
        held, s = every(), torch.cuda.Stream()
        call(s)
        s.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(held, every()))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        for k in range(3):
            zd.mul_(1.25)
            td[k] = -100
            graph.replay()
            torch.cuda.synchronize()
            got = every()
            call()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(got, every()))


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [135_168, 147_455, 163_841, 250_007])
def test_rows_in_pieces(vocab, kind):
    """Rows that no workgroup holds: targets at every piece's ends, wherever the rows begin, pieces without a logit that
    is not -infinity, rows that do not count between them."""
    dtype = TYPES[kind]
    size = torch.empty(0, dtype=dtype).element_size()
    piece = 32_768 // size
    rows = 2 * (vocab // piece) + 3
    z, t = inputs(rows, vocab, dtype)
    for i in range(rows - 3):
        t[i] = min(vocab - 1, (i // 2 + 1) * piece - 1 + i % 2 - (i % 3) * 5)
    t[rows - 3], t[rows - 2], t[rows - 1] = vocab - 1, -100, 0
    z[1, :piece + 70], z[2, -3 * piece:], z[rows - 1, 1:] = -float("inf"), -float("inf"), -float("inf")
    t[1], t[2] = vocab - 9, 3
    for gap, dgap, shift, mean in ((0, 0, 0, True), (7, 3, 1, False)):
        c = config(rows, vocab, dtype, gap=gap, dgap=dgap, mean=mean, scale=300.0)
        zw = torch.where(z == -float("inf"), torch.full((), -1e4, dtype=dtype), z)     # as good as -infinity: e^-9000 is 0
        got = run(z, t, c, shift=shift)
        check(got, zw, t, c)
        assert got[0][rows - 1].item() == 0.0 and bool((got[3][1, :piece + 70] == 0).all())
        again = run(z, t, config(rows, vocab, dtype, gap=gap, dgap=gap, mean=mean, scale=300.0), shift=shift, in_place=True)
        for a, b in zip(got, again):
            assert torch.equal(a, b)
        alone = run(z, t, c, grad=False, shift=shift)
        for a, b in zip(got[:3], alone[:3]):
            assert torch.equal(a, b)


def test_pieces_in_a_graph_and_many_rows():
    """More rows than a workgroup counts itself, replayed."""
    rows, vocab = 4_200, 66_000
    z = torch.randn((rows, vocab), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    t = torch.randint(-1, vocab, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(4))
    c = config(rows, vocab, torch.float32)
    dz, loss, total = torch.empty_like(z), torch.empty(rows, device="cuda"), torch.empty(1, device="cuda")
    count = torch.empty(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(E.ea_token_loss_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    E.ea_token_loss(c, z, t, loss, total, count, dz, ws)
    kept = [v.clone() for v in (loss, total, count, dz[::50])]
    assert count.item() == int((t >= 0).sum())
    few = slice(0, rows, 700)
    want = L.Loss(z[few].double().cpu(), t[few].cpu(), 1.0, False)
    R.within(loss[few], want.loss, want.loss_bound, "loss")
    # the gradient's factor is 1 / count: two roundings more
    R.within(dz[few], want.dz / count.item(), want.dz_bound / count.item() + 2 * U32 * want.dz.abs() / count.item() + 2.0 ** -140,
             "dlogits")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        E.ea_token_loss(c, z, t, loss, total, count, dz, ws)
    for _ in range(3):
        for v in (loss, total, count, dz, ws):
            v.view(torch.uint8).fill_(0xA5)
        graph.replay()
        assert all(map(torch.equal, (loss, total, count, dz[::50]), kept))
        torch.cuda.synchronize()
