"""Plain implementations, in 64 bits on the CPU, of the operators beside the round,
and the error bounds that the kernels' 32-bit operations allow."""
import numpy as np
import torch

U32 = 2.0 ** -24                         # rounding of one binary32 operation, relative
U16 = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 0.0}
TINY = 2.0 ** -140                       # slack for results among the subnormal numbers
BLOCK = 256


def f32(x):
    return float(np.float32(x))


class Step:
    """One AdamW step in 64 bits on float64 inputs, with the bounds of a 32-bit step beside each result."""

    def __init__(self, p, g, m, v, t, lr, beta1, beta2, eps, wd=0.0, lr_scale=1.0, gscale=1.0):
        lr, b1, b2, eps = f32(lr) * f32(lr_scale), f32(beta1), f32(beta2), f32(eps)
        wd = f32(wd)
        g = g * f32(gscale)
        self.m = b1 * m + (1 - b1) * g
        self.v = b2 * v + (1 - b2) * g * g
        self.root = self.v.sqrt()
        den = self.root / (1 - b2 ** t) ** 0.5 + eps
        step = lr / (1 - b1 ** t)
        self.p = p * (1 - lr * wd) - step * self.m / den
        # m: four roundings (g, two products, the sum) and one of 1 - beta1; v: three of g g and its factor, two of
        # b2 v, the sum, and one of 1 - beta2; the root halves v's and adds its own
        size = b1 * m.abs() + (1 - b1) * g.abs()
        self.m_bound = 5 * U32 * size + TINY
        self.v_bound = 7 * U32 * self.v + TINY
        self.root_bound = 5 * U32 * self.root + TINY ** 0.5
        # den: its root, the factor, two operations (8); the quotient and the product with the step (3); p's product
        # and the difference (3); m's own error over den
        self.p_bound = 4 * U32 * p.abs() + step * (17 * U32 * size) / den + TINY


def within(got, want, bound, what, extra=0.0):
    got = got.detach().cpu().double().reshape(-1)
    want, bound = want.reshape(-1), (bound + extra * want.abs()).reshape(-1)
    off = (got - want).abs()
    bad = ~(off <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} out of bounds, first at " \
        f"{int(bad.nonzero()[0])}: {got[bad][0]} for {want[bad][0]}, bound {bound[bad][0]}"


# ---- E4M3 codes with a scale per block, from the format's definition -----------------


def e4m3_values():
    """The value of each of the 256 codes (OCP 8-bit floating point E4M3: bias 7, no infinities)."""
    c = np.arange(256)
    e, f = (c >> 3) & 15, c & 7
    x = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * 2.0 ** (e - 7.0))
    x = np.where((c & 127) == 127, np.nan, x)
    return np.where(c >> 7 == 1, -x, x)


VALUES = e4m3_values()
POSITIVE = VALUES[:127]                  # increasing, 0 to 448


def nearest_code(y):
    """Codes of float64 values in [-448, 448], ties to the even code."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(POSITIVE, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    down, up = a - POSITIVE[lo], POSITIVE[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def decode(codes, scales):
    """float64 values of a tensor's uint8 codes."""
    x = VALUES[codes.reshape(-1)]
    return torch.from_numpy(x * np.repeat(scales.astype(np.float64), BLOCK)[:x.size])


def pad(x):
    n = -(-x.size // BLOCK) * BLOCK
    return np.concatenate([x.reshape(-1), np.zeros(n - x.size, x.dtype)]).reshape(-1, BLOCK)


def encode32(x, roots, u=None):
    """Codes and scales of float32 values, the steps of the header in binary32."""
    n, x = x.size, pad(x.astype(np.float32))
    one, top = np.float32(1), np.abs(x).max(1)
    scale = top * (one / np.float32(448))
    scale[scale < np.float32(2.0 ** -126)] = 0
    with np.errstate(divide="ignore", invalid="ignore"):
        y = np.where(scale[:, None] > 0, x * (one / scale)[:, None], np.float32(0))
    a = np.abs(y)
    if u is not None:
        u = pad(u)
        up = ((a.view(np.uint32) + ((u << np.uint32(4)) | np.uint32(8))) & np.uint32(0xFFF00000)).view(np.float32)
        low = np.floor(a * np.float32(512) + (u.astype(np.float32) + np.float32(0.5)) * np.float32(2.0 ** -16))
        a = np.where(a < np.float32(2.0 ** -6), low * np.float32(2.0 ** -9), up)
    code = nearest_code(np.copysign(np.minimum(a, np.float32(448)), y).astype(np.float64))
    if roots:
        code = np.where(((code & 127) == 0) & (x > 0) & (scale[:, None] > 0), code | 1, code).astype(np.uint8)
    return code.reshape(-1)[:n], scale


def philox_words(seed, t, stream, n, first=0):
    """The 32-bit word of each of n elements from element 4 * first: word k & 3 of Philox4x32-10 at counter
    (k >> 2, t, stream)."""
    m = np.uint64(0xFFFFFFFF)
    quad = np.arange(first, first + (n + 3) // 4, dtype=np.uint64)
    x, y = quad & m, quad >> np.uint64(32)
    z, w = np.full_like(quad, t), np.full_like(quad, stream)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        a, b = x * np.uint64(0xD2511F53), z * np.uint64(0xCD9E8D57)
        x, y, z, w = (b >> np.uint64(32)) ^ y ^ np.uint64(k0), b & m, (a >> np.uint64(32)) ^ w ^ np.uint64(k1), a & m
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack([x, y, z, w], 1).reshape(-1)[:n].astype(np.uint32)


def adamw32(p, g, m, v, t, lr, beta1, beta2, eps, wd=0.0, lr_scale=1.0, gscale=1.0):
    """m, the root of v, v and p of a step, each operation in binary32, on float32 arrays."""
    f = np.float32
    lr = float(f(lr)) * float(f(lr_scale))
    b1, b2 = float(f(beta1)), float(f(beta2))
    g = g * f(gscale)
    m = m * f(b1) + g * f(1 - b1)
    v = v * f(b2) + (g * g) * f(1 - b2)
    r = np.sqrt(v)
    den = r * f(1 / np.sqrt(1 - b2 ** t)) + f(eps)
    p = p * f(1 - lr * float(f(wd))) - (m / den) * f(lr / (1 - b1 ** t))
    return m, r, v, p


# ---- embedding -------------------------------------------------------------------------


def lookup64(table, ids, scale):
    known = (ids >= 0) & (ids < table.shape[0])
    rows = table.double()[ids.long().clamp(0, table.shape[0] - 1)] * f32(scale)
    return torch.where(known[:, None], rows, torch.zeros_like(rows))


def embed_grad64(ids, dx, vocab, scale, padding=-1, base=None):
    """The gradient in 64 bits, and the sum of its terms' magnitudes (with the number of terms) for error bounds."""
    keep = (ids >= 0) & (ids < vocab) & (ids != padding)
    at = ids[keep].long()
    d = dx.double()[keep] * f32(scale)
    total = torch.zeros((vocab, dx.shape[1]), dtype=torch.float64)
    size = total.clone()
    total.index_add_(0, at, d)
    size.index_add_(0, at, d.abs())
    count = torch.zeros(vocab, dtype=torch.float64).index_add_(0, at, torch.ones(len(at), dtype=torch.float64))
    if base is not None:
        total = total + base.double()
        size = size + base.double().abs()
    return total, size, count
