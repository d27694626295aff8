"""The token loss over more rows than a launch has workgroups, so that each takes several in turn, counted and not: rows that
are written where they were read while the next ones are on their way.  Equal logits, whose sum is exact."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402
import paper_2205_14473_amd as E  # noqa: E402
import train_util as R  # noqa: E402
from layer_util import TYPES, U32  # noqa: E402


def config(rows, vocab, kind, gap=0, mean=False, scale=1.0):
    return E.TokenLoss(rows=rows, vocab=vocab, logits_stride=vocab + gap, dlogits_stride=vocab + gap, scale=scale,
                       type=E.ea_type(kind), index_bits=64, reduction=E.EA_REDUCE_MEAN if mean else E.EA_REDUCE_SUM)


def run(c, z, t, dz):
    loss, total = torch.empty(c.rows, device="cuda"), torch.empty(1, device="cuda")
    count = torch.empty(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(E.ea_token_loss_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    E.ea_token_loss(c, z, t, loss, total, count, dz, ws)
    return loss, total, count


# vocabularies (binary32; twice as many of 16 bits) held by 1, 4, 8 and 16 waves, and in pieces; rows over the
# workgroups of the launch: 2,048 of four rows, 1,024, 512, 256
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", [(8195, 500), (17_000, 301), (2100, 4500), (1300, 21_000), (700, 34_000), (300, 70_001)])
@pytest.mark.parametrize("every", [3, 2])
def test_rows_in_turn(rows, vocab, kind, every):
    """Every second or third target does not count, NaN in its row; a workgroup's next row is 256 to 8,192 further on, so with
    3 they take turns, and with 2 a workgroup has rows of one kind only."""
    dtype = TYPES[kind]
    vocab *= 1 if kind == "f32" else 2
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    z = (torch.randn((rows, vocab), device="cuda", generator=gen) * 3).to(dtype)
    t = torch.randint(0, vocab, (rows,), device="cuda", generator=gen)
    t[::every] = -100
    z[::every, ::2] = float("nan")
    for gap in (0, 3):
        _, zd = L.spaced(z, vocab + gap, dtype)
        flat, dz = L.spaced((rows, vocab), vocab + gap, dtype)
        c = config(rows, vocab, dtype, gap, scale=300.0)
        apart = run(c, zd, t, dz)
        assert torch.equal(zd.contiguous().view(torch.uint8), z.view(torch.uint8)) and L.guards_kept(flat, dz)
        some = torch.cat([torch.arange(0, rows, rows // 40), torch.arange(rows - 8, rows)])
        want = L.Loss(torch.where(z[some].isnan(), 0.0, z[some].double()).cpu(), t[some].cpu(), 300.0, False)
        R.within(apart[0][some], want.loss, want.loss_bound, "loss")
        R.within(dz[some], want.dz, want.dz_bound + L.rounding(want.dz, dtype), "dlogits")
        assert apart[2].item() == rows - len(range(0, rows, every))
        assert bool((dz[::every] == 0).all()) and bool((apart[0][::every] == 0).all())
        assert bool(dz.isfinite().all())
        inside = run(c, zd, t, zd)
        for a, b in zip(apart + (dz,), inside + (zd,)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 7, 511, 513, 1025, 4097, 8193, 16_385, 30_001, 50_257, 65_537, 70_000, 131_073, 140_001, 250_007])
def test_equal_logits(vocab, kind):
    """Every exponential is 1, and their sum, the vocabulary, exact: the loss is its logarithm (two units at most), each
    gradient one quotient; a logit lost or taken twice changes them by 1 / vocab.  log(250,007) is 12.4: 2 U32 of it, 1.5e-6,
    are well under 1 / 250,007."""
    rows, dtype = 5, TYPES[kind]
    values = torch.tensor([0.0, 3.0, -40.0, 100.0, -1000.0], device="cuda")
    z = values[:, None].expand(rows, vocab).to(dtype).contiguous()
    t = torch.tensor([0, vocab - 1, vocab // 2, vocab // 3, -1], device="cuda")
    for shift, gap in ((0, 0), (1, 3)):
        _, zd = L.spaced(z, vocab + gap, dtype, shift)
        _, dz = L.spaced((rows, vocab), vocab + gap, dtype, shift)
        loss = run(config(rows, vocab, dtype, gap, scale=1024.0), zd, t, dz)[0]
        log = math.log(vocab)
        assert bool(((loss[:4].double() - log).abs() <= 2 * U32 * log).all()) and loss[4].item() == 0
        want = torch.full((4, vocab), 1024.0 / vocab, dtype=torch.float64)
        want[torch.arange(4), t[:4].cpu()] -= 1024.0
        # the quotient's rounding, the product's with 1, the difference's; then the result's
        R.within(dz[:4], want, 2 * U32 * 1024.0 / vocab + U32 * want.abs() + L.rounding(want, dtype), "dlogits")
