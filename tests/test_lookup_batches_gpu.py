"""Lookups of whole batches, on both sides of where a group of lanes takes four tokens: each element is one
product rounded to binary32, then to the rows' type, so the bits are those of the same on the CPU."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402
import test_embed_gpu as T  # noqa: E402


@pytest.mark.parametrize("table,x", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f16"), ("f16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n,vocab,dim", [(4095, 300, 769), (4096, 300, 768), (4097, 300, 771), (4099, 90, 1030),
                                         (8193, 70_000, 257), (30_001, 500, 63), (65_538, 1000, 50), (65_537, 7, 97)])
@pytest.mark.parametrize("gaps", [(0, 0, 0), (3, 5, 1)])
def test_batches(n, vocab, dim, table, x, gaps):
    tgap, xgap, shift = gaps
    gen = torch.Generator().manual_seed(n)
    tv = torch.randn((vocab, dim), generator=gen).to(T.TYPES[table])
    _, t = T.rows(vocab, dim, tgap, T.TYPES[table], tv, shift)
    flat, out = T.rows(n, dim, xgap, T.TYPES[x], shift=shift)
    ids = T.make_ids(n, vocab, "outside")
    c = T.config(n, vocab, dim, T.TYPES[table], T.TYPES[x], 1.7, bits=64 if n % 2 else 32, tgap=tgap, xgap=xgap)
    E.ea_embed_lookup(c, t, ids.to(torch.int64 if n % 2 else torch.int32).cuda(), out)
    known = (ids >= 0) & (ids < vocab)
    rows = tv.float()[ids.clamp(0, vocab - 1)] * torch.tensor(1.7)
    want = torch.where(known[:, None], rows, torch.zeros(())).to(T.TYPES[x])
    assert torch.equal(out.cpu(), want)
    assert T.gaps_kept(flat, n, dim, xgap, shift)
