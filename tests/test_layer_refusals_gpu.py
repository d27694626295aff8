"""Calls that the binding refuses: wrong types, shapes, strides and sizes of device tensors and workspaces that are too small,
host tensors among them. Nothing is launched and nothing written."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402

ROWS, DIM, BATCH, LENGTH = 6, 8, 2, 300


def fill(*shape, dtype=torch.float32):
    return torch.full(shape, 5, dtype=dtype, device="cuda")


def calls():
    """name -> (function, its tensors in order; a tensor's name may be given another)."""
    like = dict(x_stride=DIM, y_stride=DIM)
    norm = E.LayerNorm(rows=ROWS, dim=DIM, eps=1e-5, **like)
    drop = E.Dropout(rows=ROWS, dim=DIM, p=0.5, **like)
    rec = E.Recurrence(batch=BATCH, length=LENGTH, dim=DIM, g_stride=DIM, gate=1, **like)
    loss = E.TokenLoss(rows=ROWS, vocab=DIM, logits_stride=DIM, dlogits_stride=DIM, scale=1.0, index_bits=64)
    rows, vec, each = (ROWS, DIM), (DIM,), (ROWS,)
    steps, ends, saved = (BATCH, LENGTH, DIM), (BATCH, DIM), (BATCH, -(-LENGTH // 64), DIM)

    def ws(n):
        return fill(n, dtype=torch.uint8)

    return {
        "norm": (lambda x, w, b, y, m, r: E.ea_layer_norm(norm, x, w, b, y, m, r),
                 dict(x=fill(*rows), weight=fill(*vec), bias=fill(*vec), y=fill(*rows), mean=fill(*each), rstd=fill(*each))),
        "norm_grad": (lambda x, dy, w, m, r, a, dx, dw, db, s: E.ea_layer_norm_grad(norm, x, dy, w, m, r, a, dx, dw, db, False, s),
                      dict(x=fill(*rows), dy=fill(*rows), weight=fill(*vec), mean=fill(*each), rstd=fill(*each), add=fill(*rows),
                           dx=fill(*rows), dweight=fill(*vec), dbias=fill(*vec), workspace=ws(E.ea_layer_norm_workspace_bytes(norm)))),
        "drop": (lambda x, r, y: E.ea_dropout(drop, 1, x, r, y), dict(x=fill(*rows), residual=fill(*rows), y=fill(*rows))),
        "drop_grad": (lambda dy, dx: E.ea_dropout_grad(drop, 1, dy, dx), dict(dy=fill(*rows), dx=fill(*rows))),
        "rec": (lambda g, x, h, n, y, s, e, w: E.ea_recurrence(rec, g, x, h, n, y, s, e, w),
                dict(g=fill(*steps), x=fill(*steps), h0=fill(*ends), lengths=fill(BATCH, dtype=torch.int32), y=fill(*steps),
                     states=fill(*saved), h_last=fill(*ends), workspace=ws(E.ea_recurrence_workspace_bytes(rec)))),
        "rec_grad": (lambda g, x, s, n, dy, d, dg, dx, d0, w: E.ea_recurrence_grad(rec, g, x, s, n, dy, d, dg, dx, d0, w),
                     dict(g=fill(*steps), x=fill(*steps), states=fill(*saved), lengths=fill(BATCH, dtype=torch.int32),
                          dy=fill(*steps), dh_last=fill(*ends), dg=fill(*steps), dx=fill(*steps), dh0=fill(*ends),
                          workspace=ws(E.ea_recurrence_workspace_bytes(rec)))),
        "loss": (lambda z, t, l, tot, c, dz, w: E.ea_token_loss(loss, z, t, l, tot, c, dz, w),
                 dict(logits=fill(*rows), targets=fill(ROWS, dtype=torch.int64), loss=fill(*each), total=fill(1),
                      count=fill(1, dtype=torch.int32), dlogits=fill(*rows),
                      workspace=ws(E.ea_token_loss_workspace_bytes(loss)))),
    }


def wrongs(name, t):
    """Tensors that do not fit in t's place."""
    if name == "workspace":
        return [t[:-1]]
    out = [t.to(torch.float16 if t.dtype != torch.float16 else torch.float32), t[:-1] if t.shape[0] > 1 else t[:0], t.cpu()]
    if t.dim() > 1:
        out += [t[..., :-1], t.transpose(-1, -2).contiguous().transpose(-1, -2), t.flatten()[:-8]]
    elif t.shape[0] > 1:
        out += [t.repeat(2)[::2]]
    return out


@pytest.mark.parametrize("name", ["norm", "norm_grad", "drop", "drop_grad", "rec", "rec_grad", "loss"])
def test_wrong_tensors(name):
    call, args = calls()[name]
    for arg, t in args.items():
        for bad in wrongs(arg, t):
            with pytest.raises(ValueError):
                call(*{**args, arg: bad}.values())
    torch.cuda.synchronize()
    for arg, t in args.items():
        assert bool((t == 5).all()), arg
    call(*args.values())                               # as they are, they are taken
    torch.cuda.synchronize()
