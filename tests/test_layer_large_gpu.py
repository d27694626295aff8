"""Arrays of 64 MiB and more, whose results go past the caches: the same bits as in parts that are smaller, nothing
between the rows written."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402
import paper_2205_14473_amd as E  # noqa: E402

LARGE = 64 << 20
KINDS = ["f32", "bf16", "f16"]


def rows_of(dim, dtype):
    """Rows of a little more than LARGE bytes, two parts of which are smaller."""
    n = LARGE // (dim * torch.empty(0, dtype=dtype).element_size()) + 3
    return n + n % 2


def rand(rows, dim, dtype, seed):
    return torch.randn((rows, dim), device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(dtype)


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dim", [5, 64, 256, 1001, 4096, 8190, 20_001])
def test_norm(dim, kind):
    dtype = L.TYPES[kind]
    rows, code, gap = rows_of(dim, dtype), E.ea_type(dtype), 3
    x, dy, w, b = rand(rows, dim, dtype, 1), rand(rows, dim, dtype, 2), torch.rand(dim, device="cuda"), torch.rand(dim, device="cuda")

    def run(at, n):
        c = E.LayerNorm(rows=n, dim=dim, x_stride=dim, y_stride=dim + gap, eps=1e-5, x_type=code, y_type=code, w_type=E.EA_F32)
        flat, y = L.spaced((n, dim), dim + gap, dtype)
        _, d = L.spaced(dy[at:at + n], dim + gap, dtype)
        mean, rstd, dx = torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, dim), dtype=dtype, device="cuda")
        E.ea_layer_norm(c, x[at:at + n], w, b, y, mean, rstd)
        E.ea_layer_norm_grad(c, x[at:at + n], d, w, mean, rstd, x[at:at + n], dx, None, None, False, None)
        assert L.guards_kept(flat, y)
        return y, dx

    whole = run(0, rows)
    for at in (0, rows // 2):
        for a, b_ in zip(whole, run(at, rows // 2)):
            assert same(a[at:at + rows // 2], b_)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("gap", [0, 3])
def test_dropout(kind, gap):
    dtype, dim = L.TYPES[kind], 1001
    rows, code = rows_of(dim, dtype), E.ea_type(dtype)
    x, res = rand(rows, dim, dtype, 1), rand(rows, dim, dtype, 2)

    def run(n):
        c = E.Dropout(rows=n, dim=dim, x_stride=dim, y_stride=dim + gap, p=0.3, x_type=code, y_type=code, site=1, seed=5)
        flat, y = L.spaced((n, dim), dim + gap, dtype)
        _, r = L.spaced(res[:n], dim + gap, dtype)
        dx = torch.empty((n, dim), dtype=dtype, device="cuda")
        E.ea_dropout(c, 9, x[:n], r, y)
        E.ea_dropout_grad(c, 9, r, dx)
        assert L.guards_kept(flat, y)
        return y, dx

    for a, b in zip(run(rows), run(rows // 2)):
        assert same(a[:rows // 2], b)


@pytest.mark.parametrize("gate", [0, 1])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("batch, length, dim", [(65_600, 1, 520), (514, 100, 700), (6, 6000, 1001)])
def test_recurrence(batch, length, dim, kind, gate):
    dtype = L.TYPES[kind]
    code, gap = E.ea_type(dtype), 3
    rows, step = batch * length, -(-batch // 3)
    assert rows * dim * 2 >= LARGE > step * length * dim * 4
    x, g, dy = (rand(rows, dim, dtype, k) for k in range(3))
    g = g if gate else (g.float() * 0.2).to(dtype)
    lengths = torch.tensor([max(0, length - 37 * (k % 3)) for k in range(batch)], dtype=torch.int32, device="cuda")

    def run(at, n):
        c = E.Recurrence(batch=n, length=length, dim=dim, x_stride=dim, g_stride=dim, y_stride=dim + gap, gate=gate,
                         x_type=code, g_type=code)
        here = slice(at * length, (at + n) * length)
        flat, y = L.spaced((n * length, dim), dim + gap, dtype)
        _, d = L.spaced(dy[here], dim + gap, dtype)
        states = torch.empty(E.ea_recurrence_states_bytes(c) // 4, device="cuda")
        ws = torch.empty(E.ea_recurrence_workspace_bytes(c), dtype=torch.uint8, device="cuda")
        dg, dx = torch.empty_like(g[here]), torch.empty_like(x[here])
        E.ea_recurrence(c, g[here], x[here], None, lengths[at:at + n], y, states, None, ws)
        E.ea_recurrence_grad(c, g[here], x[here], states, lengths[at:at + n], d, None, dg, dx, None, ws)
        assert L.guards_kept(flat, y)
        return y, dg, dx

    whole = run(0, batch)
    for at in range(0, batch, step):
        n = min(step, batch - at)
        for a, b in zip(whole, run(at, n)):
            assert same(a[at * length:(at + n) * length], b)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("vocab", [7, 300, 2_003, 8_192, 30_001, 60_000, 140_001])
def test_loss(vocab, kind):
    dtype = L.TYPES[kind]
    rows, code, gap = rows_of(vocab, dtype), E.ea_type(dtype), 3
    z = rand(rows, vocab, dtype, 1)
    t = torch.randint(-1, vocab, (rows,), device="cuda", generator=torch.Generator(device="cuda").manual_seed(2))

    def run(at, n):
        c = E.TokenLoss(rows=n, vocab=vocab, logits_stride=vocab, dlogits_stride=vocab + gap, scale=0.5, type=code,
                        index_bits=64, reduction=E.EA_REDUCE_SUM)
        flat, dz = L.spaced((n, vocab), vocab + gap, dtype)
        loss, total = torch.empty(n, device="cuda"), torch.empty(1, device="cuda")
        ws = torch.empty(E.ea_token_loss_workspace_bytes(c), dtype=torch.uint8, device="cuda")
        E.ea_token_loss(c, z[at:at + n], t[at:at + n], loss, total, None, dz, ws)
        assert L.guards_kept(flat, dz)
        return loss, dz

    whole = run(0, rows)
    for at in (0, rows // 2):
        for a, b in zip(whole, run(at, rows // 2)):
            assert same(a[at:at + rows // 2], b)
