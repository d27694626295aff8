"""Plain implementations, in 64 bits on the CPU, of the layers' operators, and the error bounds that the kernels'
32-bit operations allow: U32 for each rounding of an operation, 2 U32 where a function may be a unit off."""
import numpy as np
import torch

import train_util as R
from train_util import U16, U32  # noqa: F401

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LEAST = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}   # absolute, of a rounding
GUARD = 55.0


def spaced(values, stride, dtype, shift=0):
    """(the allocation, [rows, dim] of it): rows `stride` elements apart, `shift` elements into it, GUARD elsewhere.
    values: the rows, or (rows, dim) for rows of GUARD too."""
    rows, dim = values if isinstance(values, tuple) else values.shape
    flat = torch.full((shift + rows * stride + 16,), GUARD, dtype=dtype, device="cuda")
    view = flat[shift:shift + rows * stride].view(rows, stride)[:, :dim]
    if not isinstance(values, tuple):
        view.copy_(values)
    return flat, view


def guards_kept(flat, view, shift=0):
    rows, stride = view.shape[0], view.stride(0) if view.shape[0] else 1
    left = torch.ones_like(flat, dtype=torch.bool)
    if rows:
        left[shift:shift + rows * stride].view(rows, stride)[:, :view.shape[1]] = False
    return bool((flat[left] == GUARD).all())


def rounding(want, dtype):
    """Half a step of the result's type."""
    return U16[dtype] * want.abs() + LEAST[dtype]


# ---- layer norm ------------------------------------------------------------------------


def depth(dim):
    """Additions that one term of a row's sum passes through: a lane's own (16, or dim / 1024 of a long row), six
    across the wave, 16 waves."""
    return 16 + 6 + 16 + dim // 1024


class Norm:
    def __init__(self, x, w, b, eps):
        eps, n = R.f32(eps), x.shape[1]
        self.mean = x.mean(1)
        d = x - self.mean[:, None]
        var = d.square().mean(1)
        self.rstd = 1 / (var + eps).sqrt()
        self.hat = d * self.rstd[:, None]
        self.y = self.hat * w + b
        k = depth(n)
        self.mean_bound = (k + 2) * U32 * x.abs().mean(1) + 2.0 ** -140
        # squares: the difference's rounding twice, the sum's, one for 1 / n; the mean's error enters squared
        var_bound = (k + 5) * U32 * var + self.mean_bound.square() + 2 * U32 * d.abs().mean(1) * self.mean_bound
        # the sum with eps, root, reciprocal
        rel = var_bound / (2 * (var + eps)) + 6 * U32
        self.rstd_bound = rel * self.rstd
        self.y_bound = w.abs() * (self.rstd[:, None] * (self.mean_bound[:, None] + U32 * d.abs())
                                  + self.hat.abs() * (rel[:, None] + 3 * U32)) + 2 * U32 * self.y.abs() + 2.0 ** -140


class NormGrad:
    def __init__(self, x, dy, w, mean, rstd, add=None, dw=None, db=None):
        n, rows = x.shape[1], x.shape[0]
        r = rstd[:, None]
        hat = (x - mean[:, None]) * r
        q = dy * w
        first, second = q.mean(1, keepdim=True), (q * hat).mean(1, keepdim=True)
        inner = q - first - hat * second
        self.dx = r * inner
        k = depth(n)
        size = q.abs() + first.abs() + (hat * second).abs()
        # q: 1; first: its sum and 1 / n; second: the sum of products of q and hat (1 + 2); hat second: 3; two differences
        self.dx_bound = r * ((k + 3) * U32 * (q.abs().mean(1, keepdim=True))
                             + hat.abs() * (k + 6) * U32 * (q * hat).abs().mean(1, keepdim=True) + 6 * U32 * size) \
            + U32 * self.dx.abs() + 2.0 ** -140
        if add is not None:
            self.dx = self.dx + add
            self.dx_bound = self.dx_bound + U32 * self.dx.abs()
        self.dw, self.db = (dy * hat).sum(0), dy.sum(0)
        self.dw_bound = (rows + 4) * U32 * (dy * hat).abs().sum(0) + 2.0 ** -140
        self.db_bound = (rows + 2) * U32 * dy.abs().sum(0) + 2.0 ** -140
        if dw is not None:
            self.dw, self.db = self.dw + dw, self.db + db
            self.dw_bound = self.dw_bound + U32 * self.dw.abs()
            self.db_bound = self.db_bound + U32 * self.db.abs()


# ---- dropout ---------------------------------------------------------------------------


def kept(seed, t, site, rows, dim, p):
    """(which elements stay, [rows, dim]; the factor on them): from the 32-bit words of the generator."""
    n = rows * dim
    words = R.philox_words(seed, t, site, -(-n // 8) * 4)
    halves = np.stack([words & np.uint32(0xFFFF), words >> np.uint32(16)], 1).reshape(-1)[:n]
    limit = int(np.rint(np.float64(np.float32(p)) * 65536))
    factor = 65536 / (65536 - limit) if limit < 65536 else 0.0
    return torch.from_numpy(halves.astype(np.int64) >= limit).view(rows, dim), np.float32(factor).item()


def dropout(x, residual, keep, factor, dtype):
    """The bits of the operation: one product and one sum in binary32, one rounding to the result's type."""
    v = torch.where(keep, x.float() * torch.tensor(factor), torch.zeros(()))
    if residual is not None:
        v = residual.float() + v
    return v.to(dtype)


# ---- recurrence --------------------------------------------------------------------------


def gates(g, gate):
    return (g, torch.ones_like(g)) if gate == 0 else (torch.sigmoid(g), torch.sigmoid(-g))


class Recurrence:
    """Step by step; bounds by the same steps over magnitudes: a term that passes t steps has been multiplied by t
    gates, each wrong by at most (6 + 2 |g|) U32 (the exponential's argument, three functions of a unit), and rounded
    three times a step at most (its product, its sum, a fold)."""

    def __init__(self, g, x, h0, lengths, gate):
        b, n, dim = x.shape
        self.a, self.w = gates(g, gate)
        self.slack = (9 + (2 * g.abs() if gate else 0 * g)) * U32
        h, size, off = h0.clone(), h0.abs(), torch.zeros_like(h0)
        self.before, self.before_off = torch.zeros_like(x), torch.zeros_like(x)
        self.y, self.bound = torch.zeros_like(x), torch.zeros_like(x)
        blocks = -(-n // 64)
        self.states, self.states_bound = torch.zeros(b, blocks, dim, dtype=x.dtype), torch.zeros(b, blocks, dim, dtype=x.dtype)
        for t in range(n):
            if t % 64 == 0:
                self.states[:, t // 64], self.states_bound[:, t // 64] = h, off
            on = (t < lengths)[:, None]
            self.before[:, t], self.before_off[:, t] = h, off
            v = self.w[:, t] * x[:, t]
            a = self.a[:, t]
            new_size = a.abs() * size + v.abs()
            new_off = a.abs() * off + self.slack[:, t] * new_size + 2.0 ** -140
            h, size, off = (torch.where(on, p, q) for p, q in ((a * h + v, h), (new_size, size), (new_off, off)))
            self.y[:, t], self.bound[:, t] = torch.where(on, h, 0 * h), torch.where(on, off, 0 * off)
        self.h_last, self.h_last_bound = h, off


class RecurrenceGrad:
    def __init__(self, g, x, h0, lengths, gate, dy, dh_last):
        f = Recurrence(g, x, h0, lengths, gate)
        b, n, dim = x.shape
        e, size, off = dh_last.clone(), dh_last.abs(), torch.zeros_like(dh_last)
        self.dg, self.dx = torch.zeros_like(x), torch.zeros_like(x)
        self.dg_bound, self.dx_bound = torch.zeros_like(x), torch.zeros_like(x)
        for t in range(n - 1, -1, -1):
            on = (t < lengths)[:, None]
            a, w, k, h, xt = f.a[:, t], f.w[:, t], f.slack[:, t], f.before[:, t], x[:, t]
            d = dy[:, t] + e
            d_size = dy[:, t].abs() + size
            d_off = off + U32 * d_size
            dx, dx_off = w * d, w * (d_off + k * d.abs())
            if gate == 0:
                dg, dg_off = d * h, d_off * h.abs() + d.abs() * f.before_off[:, t] + U32 * (d * h).abs()
            else:
                dg = d * (h - xt) * a * w
                dg_off = a * w * (d_off * (h - xt).abs() + d.abs() * (f.before_off[:, t] + U32 * (h - xt).abs())) \
                    + 2 * k * dg.abs()
            for to, v in ((self.dx, dx), (self.dx_bound, dx_off), (self.dg, dg), (self.dg_bound, dg_off)):
                to[:, t] = torch.where(on, v, 0 * v)
            e, size, off = (torch.where(on, p, q) for p, q in ((a * d, e), (a.abs() * d_size, size),
                                                               (a.abs() * (d_off + k * d_size) + 2.0 ** -140, off)))
        self.dh0, self.dh0_bound = e, off


# ---- token loss ----------------------------------------------------------------------------


class Loss:
    def __init__(self, z, targets, scale, mean):
        rows, vocab = z.shape
        used = (targets >= 0) & (targets < vocab)
        at = targets.clamp(0, vocab - 1)[:, None]
        top = z.max(1, keepdim=True).values
        d = z - top
        e = d.exp()
        sum_ = e.sum(1, keepdim=True)
        hit = d.gather(1, at)
        zero = torch.zeros(rows, dtype=z.dtype)
        self.loss = torch.where(used, (sum_.log() - hit)[:, 0], zero)
        # an exponential: its difference, product and constant (3 |d|), the function (2); the sum: a lane's additions
        # (128, or more of a long row), six, 16
        k = 128 + 22 + vocab // 4096
        far = torch.where(d.isfinite(), d.abs(), 0 * d)
        rel = (e * (3 * far + 2)).sum(1, keepdim=True) / sum_ * U32 + k * U32
        self.loss_bound = (rel + 2 * U32 * sum_.log().abs() + U32 * hit.abs())[:, 0] + U32 * self.loss.abs() + 2.0 ** -140
        self.count = int(used.sum())
        each = 1 / max(1, self.count) if mean else 1.0
        self.total = float(self.loss.sum() * each)
        self.total_bound = float(self.loss_bound[used].sum() * each) + 2 * U32 * abs(self.total)
        factor = R.f32(scale) * each
        p = e / sum_ * factor
        self.dz = p - torch.zeros_like(p).scatter(1, at, factor)
        # the factor (1), its quotient by the sum (1), the product, the difference
        self.dz_bound = p * ((3 * far + 2) * U32 + rel + 4 * U32) + 2 * U32 * self.dz.abs() + 2.0 ** -140
        self.dz_bound += torch.zeros_like(p).scatter(1, at, U32 * abs(factor))
        for name in ("dz", "dz_bound"):
            setattr(self, name, torch.where(used[:, None], getattr(self, name), torch.zeros_like(p)))
