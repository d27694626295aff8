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

    python examples/next_token.py --optimizer adamw8 --steps 200
"""
import argparse
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2205_14473_amd as E  # noqa: E402
from paper_2205_14473_amd.state import adamw_list, allocate, init_state  # noqa: E402


class Model:
    """Parameters as views of one flat vector, as the round takes them."""

    def __init__(self, vocab, dim, hidden, batch, length, flat=None, seed=0):
        self.vocab, self.dim, self.tokens = vocab, dim, batch * length
        shapes = dict(table=(vocab, dim), w1=(dim, hidden), b1=(hidden,), w2=(hidden, vocab), b2=(vocab,))
        size = sum(math.prod(s) for s in shapes.values())
        self.flat = torch.empty(size, device="cuda") if flat is None else flat
        self.shapes, self.size = shapes, size
        self.p = self.views(self.flat)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        for name, t in self.p.items():
            fan = {"table": dim, "w1": dim, "w2": hidden}.get(name)
            t.copy_(torch.randn(t.shape, device="cuda", generator=gen) / math.sqrt(fan) if fan else torch.zeros_like(t))
        self.embed = E.Embed(tokens=self.tokens, vocab=vocab, dim=dim, table_stride=dim, x_stride=dim, padding=-1,
                             scale=math.sqrt(dim), table_type=E.EA_F32, x_type=E.EA_F32, index_bits=64)
        self.workspace = torch.empty(E.ea_embed_workspace_bytes(self.embed), dtype=torch.uint8, device="cuda")
        self.x = torch.empty((self.tokens, dim), device="cuda")

    def views(self, flat):
        out, at = {}, 0
        for name, shape in self.shapes.items():
            n = math.prod(shape)
            out[name] = flat[at:at + n].view(shape)
            at += n
        return out

    def gradients(self, ids, targets, grads):
        """The loss of a batch; every parameter's gradient is written to its view in `grads`."""
        E.ea_embed_lookup(self.embed, self.p["table"], ids, self.x)
        leaves = {k: self.p[k].detach().requires_grad_() for k in ("w1", "b1", "w2", "b2")}
        x = self.x.detach().requires_grad_()
        h = torch.tanh(x @ leaves["w1"] + leaves["b1"])
        loss = torch.nn.functional.cross_entropy(h @ leaves["w2"] + leaves["b2"], targets)
        got = torch.autograd.grad(loss, [x, *leaves.values()])
        for k, g in zip(leaves, got[1:]):
            grads[k].copy_(g)
        E.ea_embed_grad(self.embed, ids, got[0].contiguous(), grads["table"], False, self.workspace)
        return loss.detach()


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
    model = Model(args.vocab, args.dim, args.hidden, args.batch, args.length)
    data = Chain(args.vocab, args.batch, args.length)
    grads = model.views(torch.zeros(model.size, device="cuda"))
    names = list(model.p)
    tensors = adamw_list([model.p[k] for k in names], [grads[k] for k in names], state_bits=bits,
                         weight_decay=[0.0 if k in ("b1", "b2") else 0.01 for k in names])
    cfg = E.AdamW(lr=args.lr, beta1=0.9, beta2=0.99, eps=1e-8, state_bits=bits, seed=3,
                  rounding=E.EA_ROUND_STOCHASTIC if bits == 8 else E.EA_ROUND_NEAREST)
    norm, factor = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    workspace = torch.empty(E.ea_grad_norm_workspace_bytes(tensors), dtype=torch.uint8, device="cuda")
    losses = []
    for t in range(1, args.steps + 1):
        losses.append(model.gradients(*data.sample(), grads))
        E.ea_grad_norm(tensors, 1.0, 1.0, norm, factor, workspace)
        E.ea_adamw_step(cfg, t, tensors, factor)
    return torch.stack(losses).tolist()


def train_efficient(args):
    model = Model(args.vocab, args.dim, args.hidden, args.batch, args.length)
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
        losses.append(torch.stack([model.gradients(*d.sample(), g) for d, g in zip(data, rows)]).mean())
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
