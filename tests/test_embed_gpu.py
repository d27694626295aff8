"""Embedding lookup and its gradient against 64 bits: types, odd widths, row gaps, ids outside the
table, padding, one token for all, more tokens than rows and the reverse, accumulation, order of sums."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402
import train_util as R  # noqa: E402

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
GAP = 55.0


def rows(count, dim, gap, dtype, values=None, shift=0):
    """[count, dim] rows with `gap` elements of GAP between them, `shift` elements into their allocation."""
    flat = torch.full((shift + count * (dim + gap) + 8,), GAP, dtype=dtype, device="cuda")
    view = flat[shift:shift + count * (dim + gap)].view(count, dim + gap)[:, :dim]
    if values is not None:
        view.copy_(values)
    return flat, view


def gaps_kept(flat, count, dim, gap, shift=0):
    left = torch.ones_like(flat, dtype=torch.bool)
    left[shift:shift + count * (dim + gap)].view(count, dim + gap)[:, :dim] = False
    return bool((flat[left] == GAP).all())


def config(n, vocab, dim, table, x, scale=1.0, padding=-1, bits=64, tgap=0, xgap=0):
    return E.Embed(tokens=n, vocab=vocab, dim=dim, table_stride=dim + tgap, x_stride=dim + xgap, padding=padding,
                   scale=scale, table_type=E.ea_type(table), x_type=E.ea_type(x), index_bits=bits)


def make_ids(n, vocab, kind, seed=0):
    rng = np.random.default_rng(seed + n)
    if kind == "same":
        ids = np.full(n, vocab // 2)
    elif kind == "zipf":
        ids = (rng.permutation(vocab)[np.minimum(rng.zipf(1.3, n) - 1, vocab - 1)])
    elif kind == "ordered":
        ids = np.arange(n) % vocab
    else:
        ids = rng.integers(0, vocab, n)
    if kind == "outside":
        ids = np.where(rng.random(n) < 0.5, rng.choice([-100, -1, vocab, vocab + 7, 2 ** 31 - 1, -2 ** 31], n), ids)
    if kind == "nothing":
        ids = np.full(n, -1)
    return torch.from_numpy(ids.astype(np.int64))


@pytest.mark.parametrize("bits", [32, 64])
@pytest.mark.parametrize("table", TYPES)
@pytest.mark.parametrize("x", TYPES)
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (5, 7, 3), (33, 100, 64), (100, 13, 65), (9, 50, 255), (257, 300, 768),
                                         (3, 11, 1030), (2, 5, 4097)])
def test_lookup(n, vocab, dim, table, x, bits):
    gen = torch.Generator().manual_seed(dim)
    tgap, xgap, shift = (0, 0, 0) if dim % 2 == 0 else (5, 3, 1)
    tv = torch.randn((vocab, dim), generator=gen).to(TYPES[table])
    _, t = rows(vocab, dim, tgap, TYPES[table], tv, shift)
    xf, xo = rows(n, dim, xgap, TYPES[x], shift=shift)
    ids = make_ids(n, vocab, "outside" if n > 5 else "any")
    c = config(n, vocab, dim, TYPES[table], TYPES[x], 1.7, bits=bits, tgap=tgap, xgap=xgap)
    E.ea_embed_lookup(c, t, ids.to(torch.int32 if bits == 32 else torch.int64).cuda(), xo)
    want = R.lookup64(tv, ids, 1.7)
    R.within(xo, want, (R.U32 + R.U16[TYPES[x]]) * want.abs() + 2.0 ** -25, "x")
    assert gaps_kept(xf, n, dim, xgap, shift)


def run_grad(ids, dx, vocab, table, scale=1.0, padding=-1, bits=64, accumulate=False, base=None, tgap=0, xgap=0,
             shift=0):
    n, dim = dx.shape
    _, d = rows(n, dim, xgap, dx.dtype, dx, shift)
    tf, t = rows(vocab, dim, tgap, table, base, shift)
    c = config(n, vocab, dim, table, dx.dtype, scale, padding, bits, tgap, xgap)
    need = E.ea_embed_workspace_bytes(c)
    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    E.ea_embed_grad(c, ids.to(torch.int32 if bits == 32 else torch.int64).cuda(), d, t, accumulate,
                    ws[:need] if need else None)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0xA5).all()), "a write past the workspace"
    assert gaps_kept(tf, vocab, dim, tgap, shift), "a write between rows"
    return t


def check_grad(got, ids, dx, vocab, table, scale=1.0, padding=-1, base=None):
    want, size, count = R.embed_grad64(ids, dx, vocab, scale, padding, base)
    # a sum of k terms in binary32 in any order, the scale, the existing row, and the rounding to the table's type
    bound = (count[:, None] + 3) * R.U32 * size + R.U16[table] * want.abs() + (2.0 ** -25 if table != torch.float32 else 0)
    R.within(got, want, bound, "dtable")


KINDS = ["any", "same", "zipf", "ordered", "outside", "nothing"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,vocab,dim", [(1, 1, 1), (1, 1000, 16), (2, 3, 5), (31, 10, 64), (32, 4, 64), (33, 100, 66),
                                         (64, 7, 130), (129, 40, 7), (257, 9, 300), (512, 30, 20), (513, 30, 20), (500, 2000, 1100), (1000, 50, 96), (2049, 3000, 32), (5000, 700, 40),
                                         (20_000, 70_000, 8), (9000, 300_000, 4), (4096, 600, 12), (8191, 600, 12), (8193, 600, 12),
                                         (140_000, 90, 5), (262_145, 50, 4), (530_000, 1_100_000, 4), (30_000, 600_000, 3)])
def test_gradient(n, vocab, dim, kind):
    ids = make_ids(n, vocab, kind)
    dx = torch.randn((n, dim), generator=torch.Generator().manual_seed(n))
    got = run_grad(ids, dx, vocab, torch.float32, 0.7, bits=32 if n % 2 else 64)
    check_grad(got, ids, dx, vocab, torch.float32, 0.7)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("table", TYPES)
@pytest.mark.parametrize("x", TYPES)
@pytest.mark.parametrize("dim,tgap,xgap,shift", [(768, 0, 0, 0), (257, 1, 2, 1), (1500, 0, 4, 3)])
def test_gradient_types_and_strides(dim, tgap, xgap, shift, x, table, accumulate):
    n, vocab = 700, 90
    ids = make_ids(n, vocab, "zipf")
    gen = torch.Generator().manual_seed(dim)
    dx = torch.randn((n, dim), generator=gen).to(TYPES[x])
    base = torch.randn((vocab, dim), generator=gen).to(TYPES[table])
    got = run_grad(ids, dx, vocab, TYPES[table], 1.25, padding=4, accumulate=accumulate, base=base, tgap=tgap,
                   xgap=xgap, shift=shift)
    check_grad(got, ids, dx, vocab, TYPES[table], 1.25, 4, base if accumulate else None)
    if accumulate:                                  # rows without tokens keep their bits
        idle = torch.ones(vocab, dtype=torch.bool)
        idle[ids[ids != 4]] = False
        assert torch.equal(got.cpu()[idle], base[idle])


def test_padding_and_ids_outside_have_no_gradient_and_their_rows_are_not_read():
    ids = torch.tensor([3, 0, 5, -1, 3, 9, 0, 2, 2 ** 40, -2 ** 40])
    dx = torch.randn(10, 33)
    dx[[0, 2, 3, 4, 5, 8, 9]] = float("nan")        # padding 3; -1, 5, 9 and the two far ids outside a table of 5
    got = run_grad(ids, dx, 5, torch.float32, padding=3)
    want = torch.zeros(5, 33)
    want[0], want[2] = dx[1] + dx[6], dx[7]
    assert torch.equal(got.cpu(), want)
    base = torch.randn(5, 33)
    got = run_grad(ids, dx, 5, torch.float32, padding=3, accumulate=True, base=base)
    assert torch.equal(got.cpu(), torch.where(torch.tensor([1, 0, 1, 0, 0])[:, None] > 0, want + base, base))


def test_infinities_and_nan_stay_in_their_rows():
    n, vocab, dim = 3000, 40, 20
    ids = make_ids(n, vocab, "any")
    dx = torch.randn(n, dim)
    dx[100, 3], dx[200, 4], dx[300, 5] = float("nan"), float("inf"), -float("inf")
    got = run_grad(ids, dx, vocab, torch.float32).cpu()
    odd = torch.zeros(vocab, dim, dtype=torch.bool)
    for i, k in ((100, 3), (200, 4), (300, 5)):
        odd[ids[i], k] = True
    assert torch.equal(~torch.isfinite(got), odd)
    dx[~torch.isfinite(dx)] = 0
    check_grad(torch.where(odd, torch.zeros(()), got), ids, dx.masked_fill(odd[ids], 0), vocab, torch.float32)


def test_no_tokens():
    ids, dx = torch.empty(0, dtype=torch.int64), torch.empty(0, 12)
    assert not run_grad(ids, dx, 9, torch.float32).any()
    base = torch.randn(9, 12)
    assert torch.equal(run_grad(ids, dx, 9, torch.float32, accumulate=True, base=base).cpu(), base)
    E.ea_embed_lookup(config(0, 9, 12, torch.float32, torch.float32), base.cuda(), ids.cuda(), dx.cuda())


def test_gradient_is_the_lookup_s():
    """Differences: the lookup is linear, so <dx, lookup(W + D)> - <dx, lookup(W)> is <gradient, D> for
    directions D of any size."""
    n, vocab, dim, scale = 4000, 300, 24, 1.5
    ids = make_ids(n, vocab, "outside")
    gen = torch.Generator().manual_seed(1)
    dx, W = torch.randn((n, dim), generator=gen), torch.randn((vocab, dim), generator=gen)
    grad = run_grad(ids, dx, vocab, torch.float32, scale).cpu().double()
    c = config(n, vocab, dim, torch.float32, torch.float32, scale)

    def loss(table):
        x = torch.empty((n, dim), device="cuda")
        E.ea_embed_lookup(c, table.cuda(), ids.cuda(), x)
        return x.cpu().double() * dx.double()

    for seed in range(4):
        D = torch.randn((vocab, dim), generator=torch.Generator().manual_seed(10 + seed))
        got = (loss(W + D) - loss(W)).sum().item()
        want = (grad * ((W + D).double() - W.double())).sum().item()
        size = (grad.abs() * D.abs().double()).sum().item()
        assert abs(got - want) <= 60 * R.U32 * size


def test_same_bits_every_time_and_on_another_stream():
    """Sums of very different terms, in an order that only the ids fix."""
    n, vocab, dim = 30_000, 900, 36
    ids = make_ids(n, vocab, "zipf").cuda()
    dx = (torch.randn(n, dim) * 10.0 ** (torch.rand(n, 1) * 8 - 4)).cuda()
    c = config(n, vocab, dim, torch.float32, torch.float32)
    outs = []
    for stream in (None, torch.cuda.Stream(), None):
        ws = torch.randint(0, 255, (E.ea_embed_workspace_bytes(c),), dtype=torch.uint8, device="cuda")
        out = torch.full((vocab, dim), 3.0, device="cuda")
        torch.cuda.synchronize()
        E.ea_embed_grad(c, ids, dx, out, False, ws, stream)
        torch.cuda.synchronize()
        outs.append(out)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_in_a_graph_with_new_ids_every_replay():
    n, vocab, dim = 6000, 5000, 48
    ids, dx = torch.zeros(n, dtype=torch.int64, device="cuda"), torch.zeros((n, dim), device="cuda")
    c = config(n, vocab, dim, torch.float32, torch.float32)
    ws = torch.empty(E.ea_embed_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    out, eager, x = (torch.empty((vocab, dim), device="cuda") for _ in range(3))
    x = torch.empty((n, dim), device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        E.ea_embed_grad(c, ids, dx, out, False, ws)
        E.ea_embed_lookup(c, out, ids, x)
    for k in range(5):
        ids.copy_(make_ids(n, vocab, KINDS[k], seed=k))
        dx.copy_(torch.randn((n, dim), generator=torch.Generator().manual_seed(k)))
        graph.replay()
        torch.cuda.synchronize()
        got, rows_ = out.clone(), x.clone()
        E.ea_embed_grad(c, ids, dx, eager, False, ws)
        assert torch.equal(got, eager), f"replay {k}"
        E.ea_embed_lookup(c, eager, ids, x)
        assert torch.equal(rows_, x)


def test_rows_past_32_bit_offsets():
    """A table of more than 2^32 elements (2-byte ones, 9 GB): the last rows are found and written."""
    dim, vocab = 4096, (1 << 32) // 4096 + 100
    t = torch.empty((vocab, dim), dtype=torch.bfloat16, device="cuda")
    ids = torch.tensor([vocab - 1, 0, vocab - 2, vocab - 1], device="cuda")
    dx = torch.randn((4, dim), device="cuda").to(torch.bfloat16)
    c = config(4, vocab, dim, torch.bfloat16, torch.bfloat16)
    ws = torch.empty(E.ea_embed_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    t[-3:] = 1.0
    E.ea_embed_grad(c, ids, dx, t, False, ws)
    assert torch.equal(t[vocab - 2], dx[2]) and torch.equal(t[0], dx[1])
    assert torch.equal(t[vocab - 1], (dx[0].float() + dx[3].float()).to(torch.bfloat16))
    assert not t[vocab - 3].any() and not t[1].any() and not t[vocab // 2].any()
    x = torch.empty((4, dim), dtype=torch.bfloat16, device="cuda")
    E.ea_embed_lookup(c, t, ids, x)
    assert torch.equal(x, t[ids])


def test_batched_ids_and_rows_and_tensors_that_do_not_fit():
    ids = torch.randint(0, 50, (4, 6), device="cuda")
    table = torch.randn(50, 10, device="cuda")
    x, flat = torch.empty((4, 6, 10), device="cuda"), torch.empty((24, 10), device="cuda")
    c = config(24, 50, 10, torch.float32, torch.float32, 0.5)
    E.ea_embed_lookup(c, table, ids, x)
    E.ea_embed_lookup(c, table, ids.view(-1), flat)
    assert torch.equal(x.view(24, 10), flat) and torch.equal(flat, table[ids.view(-1)] * 0.5)
    ws = torch.empty(E.ea_embed_workspace_bytes(c), dtype=torch.uint8, device="cuda")
    d = torch.zeros_like(table)
    for bad, text in (((table.double(), ids, x), "float32, bfloat16 or float16"), ((table.half(), ids, x), "type"),
                      ((table[:49], ids, x), "rows"), ((table, ids.int(), x), "64-bit"), ((table, ids[:3], x), "24"),
                      ((table, ids.t(), x), "contiguous"), ((table, ids, x[:, :, :9]), "rows"),
                      ((table.t().contiguous().t(), ids, x), "strides|next to"), ((table, ids, x.cpu()), "device"),
                      ((table, ids, x.transpose(0, 1)), "strides")):
        with pytest.raises(ValueError, match=text):
            E.ea_embed_lookup(c, *bad)
        with pytest.raises(ValueError, match=text):
            E.ea_embed_grad(c, bad[1], bad[2], bad[0], False, ws)
    with pytest.raises(ValueError, match="workspace"):
        E.ea_embed_grad(c, ids, x, d, False, ws[:-1])
    with pytest.raises(E.EAError, match="workspace"):
        E.ea_embed_grad(c, ids, x, d, False, None)
    assert not d.any()


def test_what_stands_beside_the_rows_is_not_read(monkeypatch):
    """NaN between and around rows change no bit of a lookup or a gradient."""
    n, vocab, dim = 300, 40, 67
    ids = make_ids(n, vocab, "outside")
    gen = torch.Generator().manual_seed(2)
    dx, base = torch.randn((n, dim), generator=gen), torch.randn((vocab, dim), generator=gen)
    outs = []
    for beside in (55.0, float("nan")):
        monkeypatch.setattr(sys.modules[__name__], "GAP", beside)
        _, d = rows(n, dim, 5, torch.float32, dx, 3)
        _, t = rows(vocab, dim, 2, torch.float32, base, 1)
        _, x = rows(n, dim, 1, torch.float32, shift=1)
        c = config(n, vocab, dim, torch.float32, torch.float32, 1.0, 7, tgap=2, xgap=1)
        E.ea_embed_lookup(c, t, ids.cuda(), x)
        c.x_stride = dim + 5
        ws = torch.empty(E.ea_embed_workspace_bytes(c), dtype=torch.uint8, device="cuda").fill_(0xFF)
        E.ea_embed_grad(c, ids.cuda(), d, t, True, ws)
        outs.append((x.clone(), t.clone()))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])
