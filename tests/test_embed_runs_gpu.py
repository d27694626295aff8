"""The embedding's gradient over long runs of one id: sums of small integers, which binary32 holds exactly,
so that a row left out, added twice or given to another id shows in any run; and the rounding of sums of
many terms against the number of additions that one term goes through."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import test_embed_gpu as T  # noqa: E402
import train_util as R  # noqa: E402

LARGE = [(4097, 50, 24), (8193, 600, 12), (20_000, 70_000, 8), (30_000, 600_000, 3), (40_000, 31, 260), (9000, 300, 1030),
         (131_073, 5, 16), (140_000, 90, 5), (262_145, 50, 4), (530_000, 1_100_000, 4)]


@pytest.mark.parametrize("kind", ["same", "zipf", "any", "ordered", "outside"])
@pytest.mark.parametrize("n,vocab,dim", [(300, 20, 70), (512, 3, 1100), (600, 4, 33), (4096, 9, 64)] + LARGE)
def test_sums_of_small_integers_are_exact(n, vocab, dim, kind):
    """Every term is 1 to 3 or -1 to -3 and every partial sum stays under 2^24: any order gives the same bits."""
    assert 3 * n + 3 < 1 << 24
    gen = torch.Generator().manual_seed(n)
    ids = T.make_ids(n, vocab, kind)
    dx = torch.randint(1, 4, (n, dim), generator=gen) * (2 * torch.randint(0, 2, (n, dim), generator=gen) - 1)
    keep = (ids >= 0) & (ids < vocab) & (ids != 2)
    want = torch.zeros((vocab, dim), dtype=torch.int64).index_add_(0, ids[keep], dx[keep])
    base = torch.randint(-3, 4, (vocab, dim), generator=gen)
    for accumulate, kind_of_x in ((False, torch.float32), (True, torch.bfloat16)):
        got = T.run_grad(ids, dx.to(kind_of_x), vocab, torch.float32, padding=2, accumulate=accumulate, base=base.float())
        assert torch.equal(got.cpu(), (want + base if accumulate else want).float()), (accumulate, kind_of_x)


def additions(count, n, dim):
    """Additions that a term of a run of `count` tokens goes through at most: those of its chunk of the sorted
    order (8 to 64 positions, as many as leave 4096 waves), of the quarter of the chunks' rows that a wave adds,
    of the four quarters and the run's first row, and a chunk more at each end that the run does not fill."""
    chunk = 64
    while chunk > 8 and n // chunk * -(-dim // 256) < 4096:
        chunk //= 2
    return torch.minimum(count, chunk + torch.ceil((count / chunk + 2) / 4) + 5)


@pytest.mark.parametrize("kind", ["same", "zipf", "any"])
@pytest.mark.parametrize("n,vocab,dim", LARGE)
def test_rounding_of_long_sums(n, vocab, dim, kind):
    ids = T.make_ids(n, vocab, kind)
    dx = torch.randn((n, dim), generator=torch.Generator().manual_seed(n))
    got = T.run_grad(ids, dx, vocab, torch.float32, 0.7)
    want, size, count = R.embed_grad64(ids, dx, vocab, 0.7)
    bound = (additions(count, n, dim)[:, None] + 3) * R.U32 * size
    R.within(got, want, bound, "dtable")
    long = count > 1000                              # where the bound could hide a row: it is far under the sum itself
    assert (bound[long].amax(1) < 0.25 * want[long].abs().amax(1)).all()
