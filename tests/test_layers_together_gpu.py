"""A block of the layers and the loss in a row, as a model runs them, forward and back: against 64 bits, and the same
bits each time, on another stream and from a captured graph."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402
import paper_2205_14473_amd as E  # noqa: E402
from layer_util import U32  # noqa: E402

SEED, SITE, P = 77, 4, 0.125


class Run:
    """u = norm(x); h = recurrence(u as gates, x as values); y = x + dropout(h); loss(y), and the gradients: dx has
    x's as the gates' input and as the values, dy the part past the block."""

    def __init__(self, batch, length, dim, kind="f32"):
        t, code, rows = L.TYPES[kind], E.ea_type(L.TYPES[kind]), batch * length
        gen = torch.Generator(device="cuda").manual_seed(length)
        rand = lambda *n: torch.randn(n, device="cuda", generator=gen)  # noqa: E731
        self.shape, self.x, self.w, self.b = (batch, length, dim), rand(rows, dim).to(t), 1 + 0.1 * rand(dim), 0.1 * rand(dim)
        self.targets = torch.randint(-1, dim, (rows,), device="cuda", generator=gen)
        self.step = torch.tensor([3], dtype=torch.int32, device="cuda").view(torch.uint32)
        like = dict(x_stride=dim, y_stride=dim)
        self.norm = E.LayerNorm(rows=rows, dim=dim, eps=1e-5, x_type=code, y_type=code, w_type=E.EA_F32, **like)
        self.rec = E.Recurrence(batch=batch, length=length, dim=dim, g_stride=dim, gate=E.EA_GATE_SIGMOID, x_type=code,
                                g_type=code, **like)
        self.drop = E.Dropout(rows=rows, dim=dim, p=P, x_type=code, y_type=code, site=SITE, seed=SEED, **like)
        self.loss = E.TokenLoss(rows=rows, vocab=dim, logits_stride=dim, dlogits_stride=dim, scale=1.0, type=code,
                                index_bits=64, reduction=E.EA_REDUCE_MEAN)
        self.u, self.h, self.y, self.dy, self.dh, self.dg, self.dv, self.dx = (torch.empty_like(self.x) for _ in range(8))
        self.mean, self.rstd, self.each = (torch.empty(rows, device="cuda") for _ in range(3))
        self.dw, self.db, self.total = torch.empty_like(self.w), torch.empty_like(self.w), torch.empty(1, device="cuda")
        self.count = torch.empty(1, dtype=torch.int32, device="cuda")
        self.states = torch.empty(E.ea_recurrence_states_bytes(self.rec) // 4, device="cuda")
        # one workspace for all: the calls are ordered
        self.ws = torch.empty(max(E.ea_layer_norm_workspace_bytes(self.norm), E.ea_recurrence_workspace_bytes(self.rec),
                                  E.ea_token_loss_workspace_bytes(self.loss)), dtype=torch.uint8, device="cuda")

    def go(self):
        E.ea_layer_norm(self.norm, self.x, self.w, self.b, self.u, self.mean, self.rstd)
        E.ea_recurrence(self.rec, self.u, self.x, None, None, self.h, self.states, None, self.ws)
        E.ea_dropout(self.drop, 0, self.h, self.x, self.y, t_dev=self.step)
        E.ea_token_loss(self.loss, self.y, self.targets, self.each, self.total, self.count, self.dy, self.ws)
        E.ea_dropout_grad(self.drop, 0, self.dy, self.dh, t_dev=self.step)
        E.ea_recurrence_grad(self.rec, self.u, self.x, self.states, None, self.dh, None, self.dg, self.dv, None, self.ws)
        E.ea_layer_norm_grad(self.norm, self.x, self.dg, self.w, self.mean, self.rstd, self.dv, self.dx, self.dw, self.db,
                             False, self.ws)

    def results(self):
        return (self.u, self.h, self.y, self.each, self.total, self.count, self.dy, self.dg, self.dv, self.dx, self.dw,
                self.db)

    def bits(self):
        return [v.contiguous().view(torch.uint8).clone() for v in self.results()]

    def wipe(self):
        for v in (*self.results(), self.states, self.ws):
            v.view(torch.uint8).fill_(0xA5)


@pytest.mark.parametrize("batch, length, dim", [(3, 40, 33), (2, 700, 72)])
def test_against_64_bits(batch, length, dim):
    """The whole row in binary32.  A step of it rounds at most (its depth) times 2^-24 of its magnitudes: sums of a row
    (under 60 roundings), 700 steps that each keep a sigmoid's share of the errors (under 64 of them, gates of at most
    0.98), the loss's sums (under 60), the rows of dw (1,400): less than 2^11 in all, and magnitudes that exceed the
    largest result by less than 2^4: 2^-9 of it."""
    r = Run(batch, length, dim)
    r.go()
    x, w, b = (v.double().cpu().requires_grad_() for v in (r.x, r.w, r.b))
    d = x - x.mean(1, keepdim=True)
    u = d / (d.square().mean(1, keepdim=True) + L.R.f32(1e-5)).sqrt() * w + b
    a, v = torch.sigmoid(u).view(batch, length, dim), x.view(batch, length, dim)
    h, steps = torch.zeros(batch, dim, dtype=torch.float64), []
    for k in range(length):
        h = a[:, k] * h + (1 - a[:, k]) * v[:, k]
        steps.append(h)
    keep, factor = L.kept(SEED, 3, SITE, batch * length, dim, P)
    y = x + torch.where(keep, torch.stack(steps, 1).reshape(x.shape) * factor, torch.zeros_like(x))
    total = torch.nn.functional.cross_entropy(y, r.targets.cpu(), ignore_index=-1)
    got = torch.autograd.grad(total, (x, w, b))
    assert r.count.item() == int((r.targets >= 0).sum())
    for k, (own, want) in enumerate(zip((r.total, r.y, r.dx + r.dy, r.dw, r.db), (total, y, *got))):
        want = want.detach()
        assert (own.double().cpu() - want).abs().max() <= 2.0 ** 15 * U32 * want.abs().max(), k


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("batch, length, dim", [(3, 40, 33), (2, 1300, 136), (1, 5000, 64)])
def test_the_same_bits(batch, length, dim, kind):
    r = Run(batch, length, dim, kind)
    r.go()
    want = r.bits()
    assert all(torch.isfinite(v).all() for v in r.results())
    torch.cuda.synchronize()
    for stream in (None, torch.cuda.Stream()):
        with torch.cuda.stream(stream):
            r.wipe()
            r.go()
            got = r.bits()
        torch.cuda.synchronize()
        assert all(map(torch.equal, got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        r.go()
    for _ in range(3):
        r.wipe()
        graph.replay()
        assert all(map(torch.equal, r.bits(), want))
        r.go()                                         # eager work between the replays
        torch.cuda.synchronize()
    # the step is read on the device: another one drops others, eagerly and replayed alike
    r.step.view(torch.int32).fill_(4)
    graph.replay()
    replayed = r.bits()
    r.wipe()
    r.go()
    assert all(map(torch.equal, r.bits(), replayed)) and not torch.equal(replayed[2], want[2])


def test_two_graphs_share_a_workspace():
    """Captured apart, replayed in any order on one stream."""
    a, b = Run(2, 900, 70), Run(1, 1500, 130, "bf16")
    ws = torch.empty(max(a.ws.numel(), b.ws.numel()), dtype=torch.uint8, device="cuda")
    a.ws = b.ws = ws
    wants, graphs = [], []
    for r in (a, b):
        r.go()
        wants.append(r.bits())
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            r.go()
    for order in ((0, 1), (1, 0), (0, 0), (1, 1)):
        for r in (a, b):
            for v in r.results():
                v.view(torch.uint8).fill_(0xA5)
        for k in order:
            graphs[k].replay()
        for k in set(order):
            assert all(map(torch.equal, (a, b)[k].bits(), wants[k]))


def test_calls_at_once_with_a_workspace_each():
    """Two runs on two streams beside each other, each larger than the card holds at once."""
    runs = [Run(4, 6000, 512, "bf16"), Run(1, 24_000, 520, "bf16")]
    wants = []
    for r in runs:
        r.go()
        wants.append(r.bits())
        r.wipe()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        for r, s in zip(runs, streams):
            with torch.cuda.stream(s):
                r.go()
    torch.cuda.synchronize()
    for r, want in zip(runs, wants):
        assert all(map(torch.equal, r.bits(), want))
