"""The example's model with blocks of layer norm, recurrence and dropout, and the token loss: that it trains with every
optimizer, and its gradients against the same model in 64 bits, whose own gradients hold against differences."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import layer_util as L  # noqa: E402

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "next_token.py")
spec = importlib.util.spec_from_file_location("next_token", PATH)
X = importlib.util.module_from_spec(spec)
spec.loader.exec_module(X)

SIZES = dict(vocab=37, dim=16, hidden=24, batch=3)


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8", "efficient"])
def test_training_runs(optimizer):
    args = ["--optimizer", optimizer, "--steps", "12", "--vocab", "101", "--layers", "2", "--length", "150", "--batch", "4"]
    a, b = X.main(args), X.main(args)
    assert len(a) == 12 and all(math.isfinite(x) for x in a) and a == b
    assert X.main([*args, "--dropout", "0.5"]) != a


def plain(m, p, ids, targets, t, dropout, batch, length):
    """The loss in 64 bits, on the CPU."""
    x = p["table"][ids] * m.embed.scale
    for i, block in enumerate(m.blocks):
        nw, nb, wg, bg, wv = (p[k] for k in block.names)
        d = x - x.mean(1, keepdim=True)
        u = d / (d.square().mean(1, keepdim=True) + L.R.f32(1e-5)).sqrt() * nw + nb
        a = torch.sigmoid(u @ wg + bg).view(batch, length, -1)
        v = (u @ wv).view(batch, length, -1)
        h, steps = torch.zeros(batch, v.shape[2], dtype=torch.float64), []
        for k in range(length):
            h = a[:, k] * h + (1 - a[:, k]) * v[:, k]
            steps.append(h)
        keep, factor = L.kept(11, t, i, x.shape[0], x.shape[1], dropout)
        x = x + torch.where(keep, torch.stack(steps, 1).reshape(x.shape) * factor, torch.zeros_like(x))
    z = torch.tanh(x @ p["w1"] + p["b1"]) @ p["w2"] + p["b2"]
    return torch.nn.functional.cross_entropy(z, targets)


@pytest.mark.parametrize("length, layers, dropout", [(24, 2, 0.25), (150, 1, 0.0)])
def test_gradients(length, layers, dropout):
    """A path from the loss to a parameter passes sums of the tokens (at most 450), of the steps (150 a block), of the
    vocabulary, the hidden units and the channels (37 + 24 + 3 * 16 a block), under 1,000 roundings in all, of at most
    2^-24 of the magnitudes summed; those exceed the largest element of the result by less than the square root of
    their number and the block's own scale, 32 in all: 1000 * 32 * 2^-24 < 2^-9 of it."""
    m = X.Model(**SIZES, length=length, layers=layers, dropout=dropout)
    gen = torch.Generator(device="cuda").manual_seed(9)
    for k, v in m.p.items():
        v.add_(torch.randn(v.shape, device="cuda", generator=gen), alpha=0.2)
    ids, targets = X.Chain(37, 3, length).sample()
    grads = m.views(torch.full((m.size,), float("nan"), device="cuda"))
    loss = m.gradients(ids, targets, grads, 5)
    leaves = {k: v.double().cpu().requires_grad_() for k, v in m.p.items()}
    want = plain(m, leaves, ids.cpu(), targets.cpu(), 5, dropout, 3, length)
    exact = dict(zip(leaves, torch.autograd.grad(want, list(leaves.values()))))
    want = want.detach()
    assert abs(loss.item() - want) <= 2.0 ** -9 * want
    for k, g in grads.items():
        assert (g.double().cpu() - exact[k]).abs().max() <= 2.0 ** -9 * exact[k].abs().max(), k
    # differences in 64 bits: a step of 2^-12 leaves terms of its square, and the loss's roundings over the step
    with torch.no_grad():
        for k, g in exact.items():
            along = g / g.norm() + torch.randn(g.shape, dtype=torch.float64, generator=torch.Generator().manual_seed(3)) / g.numel() ** 0.5
            got = [plain(m, {**leaves, k: leaves[k] + s * along}, ids.cpu(), targets.cpu(), 5, dropout, 3, length)
                   for s in (2.0 ** -12, -2.0 ** -12)]
            slope = (g * along).sum()
            assert abs((got[0] - got[1]) * 2.0 ** 11 - slope) <= 1e-4 * abs(slope) + 1e-5, k
