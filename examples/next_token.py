"""A next-token model trained with the operators of this package, in two ways.

The model: embedding lookup with scaling, one hidden layer, a softmax over the
vocabulary; its data: sequences of a fixed random Markov chain, made here.

  --optimizer adamw | adamw8   one worker: gradients of every parameter, their
                               global norm and clip factor, one AdamW step over
                               all tensors (states in 32 or 8 bits)
  --optimizer efficient        N workers: each writes its gradients into its row
                               of the round's gradient array (the embedding's
                               through ea_embed_grad), then one Efficient-Adam
                               round with 4-bit messages

The hidden layer and the loss are torch's; the lookup, the embedding's
gradient, the norm and the steps are libea's.

With --layers N, blocks of libea's layers stand between the lookup and the hidden
layer: layer norm, gates and values (products of torch's), the gated recurrence
over each sequence, dropout with the block's input added.  The loss and its
gradient are then libea's too, and so are the gradients of all of these.

    python examples/next_token.py --optimizer adamw8 --steps 200
    python examples/next_token.py --layers 2 --dropout 0.1
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2205_14473_amd as E  # noqa: E402
from paper_2205_14473_amd.state import adamw_list, allocate, init_state  # noqa: E402


class Block:
    """x + dropout(recurrence(gates, values)) of x's layer norm, for rows of `batch` sequences of `length` tokens."""

    def __init__(self, index, dim, batch, length, dropout):
        self.names = [f"{k}{index}" for k in ("nw", "nb", "wg", "bg", "wv")]
        rows, f32 = batch * length, E.EA_F32
        self.norm = E.LayerNorm(rows=rows, dim=dim, x_stride=dim, y_stride=dim, eps=1e-5, x_type=f32, y_type=f32,
                                w_type=f32)
        self.rec = E.Recurrence(batch=batch, length=length, dim=dim, x_stride=dim, g_stride=dim, y_stride=dim,
                                gate=E.EA_GATE_SIGMOID, x_type=f32, g_type=f32)
        self.drop = E.Dropout(rows=rows, dim=dim, x_stride=dim, y_stride=dim, p=dropout, x_type=f32, y_type=f32,
                              site=index, seed=11)
        empty = lambda *n, dtype=torch.float32: torch.empty(n, dtype=dtype, device="cuda")  # noqa: E731
        self.u, self.g, self.v, self.h, self.out = (empty(rows, dim) for _ in range(5))
        self.mean, self.rstd = empty(rows), empty(rows)
        self.states = empty(E.ea_recurrence_states_bytes(self.rec) // 4)
        self.workspace = empty(max(E.ea_layer_norm_workspace_bytes(self.norm),
                                   E.ea_recurrence_workspace_bytes(self.rec)), dtype=torch.uint8)

    def forward(self, p, x, t):
        nw, nb, wg, bg, wv = (p[k] for k in self.names)
        self.x = x
        E.ea_layer_norm(self.norm, x, nw, nb, self.u, self.mean, self.rstd)
        torch.addmm(bg, self.u, wg, out=self.g)
        torch.mm(self.u, wv, out=self.v)
        E.ea_recurrence(self.rec, self.g, self.v, None, None, self.h, self.states, None, self.workspace)
        E.ea_dropout(self.drop, t, self.h, x, self.out)
        return self.out

    def backward(self, p, grads, d, t):
        """The gradient of x for d, that of the output; d is overwritten."""
        nw, nb, wg, bg, wv = (p[k] for k in self.names)
        dnw, dnb, dwg, dbg, dwv = (grads[k] for k in self.names)
        dh, dg, dv = torch.empty_like(d), torch.empty_like(d), torch.empty_like(d)
        E.ea_dropout_grad(self.drop, t, d, dh)
        E.ea_recurrence_grad(self.rec, self.g, self.v, self.states, None, dh, None, dg, dv, None, self.workspace)
        torch.mm(self.u.t(), dg, out=dwg)
        torch.mm(self.u.t(), dv, out=dwv)
        torch.sum(dg, 0, out=dbg)
        du = torch.mm(dg, wg.t()).addmm_(dv, wv.t())
        E.ea_layer_norm_grad(self.norm, self.x, du, nw, self.mean, self.rstd, d, d, dnw, dnb, False, self.workspace)
        return d


class Model:
    """Parameters as views of one flat vector, as the round takes them."""

    def __init__(self, vocab, dim, hidden, batch, length, flat=None, seed=0, layers=0, dropout=0.0):
        self.vocab, self.dim, self.tokens = vocab, dim, batch * length
        self.blocks = [Block(i, dim, batch, length, dropout) for i in range(layers)]
        shapes = dict(table=(vocab, dim), w1=(dim, hidden), b1=(hidden,), w2=(hidden, vocab), b2=(vocab,))
        for block in self.blocks:
            shapes.update(zip(block.names, ((dim,), (dim,), (dim, dim), (dim,), (dim, dim))))
        size = sum(math.prod(s) for s in shapes.values())
        self.flat = torch.empty(size, device="cuda") if flat is None else flat
        self.shapes, self.size = shapes, size
        self.p = self.views(self.flat)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for name, t in self.p.items():
            fan = {"table": dim, "w1": dim, "w2": hidden}.get(name, dim if name[:2] in ("wg", "wv") else None)
            t.copy_(torch.randn(t.shape, device="cuda", generator=gen) / math.sqrt(fan) if fan else
                    torch.ones_like(t) if name[:2] == "nw" else torch.zeros_like(t))
        self.embed = E.Embed(tokens=self.tokens, vocab=vocab, dim=dim, table_stride=dim, x_stride=dim, padding=-1,
                             scale=math.sqrt(dim), table_type=E.EA_F32, x_type=E.EA_F32, index_bits=64)
        self.workspace = torch.empty(E.ea_embed_workspace_bytes(self.embed), dtype=torch.uint8, device="cuda")
        self.x = torch.empty((self.tokens, dim), device="cuda")
        self.loss = E.TokenLoss(rows=self.tokens, vocab=vocab, logits_stride=vocab, dlogits_stride=vocab, scale=1.0,
                                type=E.EA_F32, index_bits=64, reduction=E.EA_REDUCE_MEAN)
        self.loss_workspace = torch.empty(E.ea_token_loss_workspace_bytes(self.loss), dtype=torch.uint8, device="cuda")

    def views(self, flat):
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = math.prod(shape)
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out

    def gradients(self, ids, targets, grads, t=0):
        """The loss of a batch; every parameter's gradient is written to its view in `grads`.  t numbers the draws of
        the dropouts."""
        E.ea_embed_lookup(self.embed, self.p["table"], ids, self.x)
        if self.blocks:
            return self.gradients_of_blocks(ids, targets, grads, t)
        leaves = {k: self.p[k].detach().requires_grad_() for k in ("w1", "b1", "w2", "b2")}
        x = self.x.detach().requires_grad_()
        h = torch.tanh(x @ leaves["w1"] + leaves["b1"])
        loss = torch.nn.functional.cross_entropy(h @ leaves["w2"] + leaves["b2"], targets)
        got = torch.autograd.grad(loss, [x, *leaves.values()])
        for k, g in zip(leaves, got[1:]):
            grads[k].copy_(g)
        E.ea_embed_grad(self.embed, ids, got[0].contiguous(), grads["table"], False, self.workspace)
        return loss.detach()


    def gradients_of_blocks(self, ids, targets, grads, t):
        p, x = self.p, self.x
        for block in self.blocks:
            x = block.forward(p, x, t)
        h = torch.addmm(p["b1"], x, p["w1"]).tanh_()
        logits = torch.addmm(p["b2"], h, p["w2"])
        total = torch.empty(1, device="cuda")
        # the logits' gradient takes their place
        E.ea_token_loss(self.loss, logits, targets, None, total, None, logits, self.loss_workspace)
        torch.mm(h.t(), logits, out=grads["w2"])
        torch.sum(logits, 0, out=grads["b2"])
        d = torch.mm(logits, p["w2"].t()) * (1 - h * h)
        torch.mm(x.t(), d, out=grads["w1"])
        torch.sum(d, 0, out=grads["b1"])
        d = torch.mm(d, p["w1"].t())
        for block in reversed(self.blocks):
            d = block.backward(p, grads, d, t)
        E.ea_embed_grad(self.embed, ids, d, grads["table"], False, self.workspace)
        return total[0]


class Chain:
    """Sequences of a Markov chain in which each token has four likely successors."""

    def __init__(self, vocab, batch, length, seed=1):
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.next = torch.randint(0, vocab, (vocab, 4), device="cuda", generator=self.gen)
        self.vocab, self.batch, self.length = vocab, batch, length

    def sample(self):
        t = torch.randint(0, self.vocab, (self.batch,), device="cuda", generator=self.gen)
        rows = [t]
        for _ in range(self.length):
            pick = torch.randint(0, 4, (self.batch,), device="cuda", generator=self.gen)
            t = self.next[t, pick]
            rows.append(t)
        seq = torch.stack(rows, 1)
        return seq[:, :-1].reshape(-1), seq[:, 1:].reshape(-1)


def train_adamw(args, bits):
    model = Model(args.vocab, args.dim, args.hidden, args.batch, args.length, layers=args.layers, dropout=args.dropout)
    data = Chain(args.vocab, args.batch, args.length)
    grads = model.views(torch.zeros(model.size, device="cuda"))
    names = list(model.p)
    tensors = adamw_list([model.p[k] for k in names], [grads[k] for k in names], state_bits=bits,
                         weight_decay=[0.0 if model.p[k].dim() == 1 else 0.01 for k in names])
    cfg = E.AdamW(lr=args.lr, beta1=0.9, beta2=0.99, eps=1e-8, state_bits=bits, seed=3,
                  rounding=E.EA_ROUND_STOCHASTIC if bits == 8 else E.EA_ROUND_NEAREST)
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    workspace = torch.empty(E.ea_grad_norm_workspace_bytes(tensors), dtype=torch.uint8, device="cuda")
    losses = []
    for t in range(1, args.steps + 1):
        losses.append(model.gradients(*data.sample(), grads, t))
        E.ea_grad_norm(tensors, 1.0, 1.0, norm, factor, workspace)
        E.ea_adamw_step(cfg, t, tensors, factor)
    return torch.stack(losses).tolist()


def train_efficient(args):
    model = Model(args.vocab, args.dim, args.hidden, args.batch, args.length, layers=args.layers, dropout=args.dropout)
    # Example 1's quantizer: to nearest, so what error feedback carries over shrinks
    q = dict(kind=E.EA_Q_DET_UNIFORM, bits=4, error_feedback=1, bucket=512)
    cfg = E.Config(d=model.size, N=args.workers, placement=E.EA_ADAM_AT_SERVER, beta1=0.9, beta2=0.99, lr=args.lr,
                   eps=1e-8, seed=3, qw=E.Quant(**q), qs=E.Quant(**q))
    buffers = allocate(cfg)
    init_state(cfg, buffers)
    buffers.x.copy_(model.flat)
    model.flat, model.p = buffers.x, model.views(buffers.x)
    rows = [model.views(buffers.g[i]) for i in range(args.workers)]
    data = [Chain(args.vocab, args.batch, args.length) for _ in range(args.workers)]
    for i, d in enumerate(data):                       # one chain, each worker with draws of its own
        d.gen.manual_seed(100 + i)
    losses = []
    for t in range(1, args.steps + 1):
        losses.append(torch.stack([model.gradients(*d.sample(), g, t * args.workers + i)
                                   for i, (d, g) in enumerate(zip(data, rows))]).mean())
        E.ea_step(cfg, t, **buffers.step_args())
    return torch.stack(losses).tolist()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--optimizer", choices=["adamw", "adamw8", "efficient"], default="adamw")
    ap.add_argument("--steps", type=int, default=100)
    ap.add_argument("--workers", type=int, default=4)
    ap.add_argument("--vocab", type=int, default=997)
    ap.add_argument("--dim", type=int, default=64)
    ap.add_argument("--hidden", type=int, default=128)
    ap.add_argument("--batch", type=int, default=32)
    ap.add_argument("--length", type=int, default=64)
    ap.add_argument("--layers", type=int, default=0, help="blocks of norm, recurrence and dropout")
    ap.add_argument("--dropout", type=float, default=0.1, help="of the blocks")
    ap.add_argument("--lr", type=float, default=None)
    args = ap.parse_args(argv)
    if args.lr is None:
        args.lr = 2e-3 if args.optimizer == "efficient" else 1e-2
    losses = train_efficient(args) if args.optimizer == "efficient" else \
        train_adamw(args, 8 if args.optimizer == "adamw8" else 32)
    for t in range(0, len(losses), max(1, len(losses) // 10)):
        print(f"step {t + 1:5d}  loss {losses[t]:.4f}")
    print(f"last loss {losses[-1]:.4f}  (uniform {math.log(args.vocab):.4f}, the chain's own {math.log(4):.4f})")
    return losses


if __name__ == "__main__":
    main()
