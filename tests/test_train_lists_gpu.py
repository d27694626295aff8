"""Lists of tensors whose caller goes on with other memory."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402
from paper_2205_14473_amd.state import adamw_list  # noqa: E402


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_reads_the_gradients_that_its_list_was_made_with(bits):
    """Storages of gradients replaced after the list was made, and memory of their size taken by others:
    the step and the norm are those of the gradients as they were."""
    outs = []
    for replaced in (False, True):
        gen = torch.Generator(device="cuda").manual_seed(1)
        ps, gs = ([torch.randn(5000, device="cuda", generator=gen) for _ in range(3)] for _ in range(2))
        tl = adamw_list(ps, gs, state_bits=bits)
        if replaced:
            gs[1].data = torch.zeros(7, device="cuda")
            gs[2].set_(torch.zeros(5000, device="cuda"))
        others = [torch.full((5000,), float("nan"), device="cuda") for _ in range(40)]
        norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
        ws = torch.empty(E.ea_grad_norm_workspace_bytes(tl), dtype=torch.uint8, device="cuda")
        E.ea_grad_norm(tl, 1.0, 1.0, norm, factor, ws)
        cfg = E.AdamW(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, state_bits=bits)
        E.ea_adamw_step(cfg, 1, tl, factor)
        outs.append([norm, factor, *ps, *tl.states, *tl.scales])
        assert len(others) == 40
    for x, y in zip(*outs):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
