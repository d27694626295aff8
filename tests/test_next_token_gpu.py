"""The example that trains a next-token model with the operators together: AdamW with states in 32 and
in 8 bits, and the Efficient-Adam round on the same gradients."""
import importlib.util
import math
import os

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "next_token.py")
spec = importlib.util.spec_from_file_location("next_token", PATH)
X = importlib.util.module_from_spec(spec)
spec.loader.exec_module(X)


@pytest.mark.parametrize("optimizer", ["adamw", "adamw8", "efficient"])
def test_training_learns_the_chain(optimizer):
    losses = X.main(["--optimizer", optimizer, "--steps", "150", "--vocab", "211"])
    assert all(math.isfinite(x) for x in losses)
    # half of the way from a uniform guess to the chain's own entropy
    assert sum(losses[-10:]) / 10 < (math.log(211) + math.log(4)) / 2, losses[-1]


def test_8_bit_states_train_as_32_bit_ones():
    a, b = (X.main(["--optimizer", k, "--steps", "100", "--vocab", "211"]) for k in ("adamw", "adamw8"))
    assert abs(sum(a[-10:]) - sum(b[-10:])) / 10 < 0.15 * sum(a[-10:]) / 10
    assert X.main(["--optimizer", "adamw8", "--steps", "100", "--vocab", "211"])[:1] == b[:1]


def test_the_model_s_gradients_by_differences():
    """Each parameter's gradient, the table's through the sorted tokens, against central differences of the
    loss along a random direction.  The loss is binary32: with a step of 2^-7 its rounding (some units of
    2^-24 of 5.3) over the two steps stays under 1e-3 and the third-order term under 1e-3 of the slope."""
    m = X.Model(211, 64, 96, 8, 32)
    ids, targets = X.Chain(211, 8, 32).sample()
    grads = m.views(torch.zeros(m.size, device="cuda"))
    scratch = m.views(torch.zeros(m.size, device="cuda"))
    m.gradients(ids, targets, grads)
    for k, p in m.p.items():
        D = torch.randn(p.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5))
        D = D / D.norm() + grads[k] / grads[k].norm()
        want, h, keep = (grads[k] * D).sum().item(), 2.0 ** -7, p.clone()
        got = []
        for s in (h, -h):
            p.copy_(keep + s * D)
            got.append(m.gradients(ids, targets, scratch).item())
            p.copy_(keep)
        assert abs((got[0] - got[1]) / (2 * h) - want) <= 1e-3 + 2e-3 * abs(want), k
