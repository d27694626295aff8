"""AdamW with 8-bit states: whole blocks of ordinary values take a shorter form than ragged ends and
unusual values.  What the two leave has to be the same, up to the bound that the header states for p."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():  # pragma: no cover - CPU-only host
    pytest.skip("needs a GPU", allow_module_level=True)

import paper_2205_14473_amd as E  # noqa: E402
import train_util as R  # noqa: E402

HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.95)


class Block8:
    """One tensor with 8-bit states in float32 and as codes, on the host."""

    def __init__(self, n, seed=1):
        rng = np.random.default_rng(seed)
        self.n, blocks = n, -(-n // 256)
        self.p = (rng.standard_normal(n) * 0.1).astype(np.float32)
        self.g = (rng.standard_normal(n) * 1e-2).astype(np.float32)
        self.cm, self.ms = R.encode32((rng.standard_normal(n) * 3e-3).astype(np.float32), False)
        self.cv, self.vs = R.encode32(np.abs(rng.standard_normal(n) * 1e-2).astype(np.float32), True)
        assert self.ms.shape == (blocks,)

    def values(self, codes, scales):
        return R.VALUES[codes].astype(np.float32) * np.repeat(scales, 256)[:self.n]

    def wanted(self, t, eps):
        """m, root, p of the step, each operation in binary32."""
        with np.errstate(over="ignore", invalid="ignore"):
            r = self.values(self.cv, self.vs)
            m, r, _, p = R.adamw32(self.p, self.g, self.values(self.cm, self.ms), r * r, t, eps=eps, **HYPER)
        return m, r, p

    def step(self, t, eps, **kw):
        """(p, codes and scales of m, codes and scales of the root) after the step on the GPU."""
        up = lambda x: torch.from_numpy(x.copy()).cuda()  # noqa: E731
        p, g, m, v, ms, vs = (up(x) for x in (self.p, self.g, self.cm, self.cv, self.ms, self.vs))
        cfg = E.AdamW(eps=eps, state_bits=8, **HYPER, **kw)
        E.ea_adamw_step(cfg, t, E.TensorList([g], p=[p], m=[m], v=[v], m_scale=[ms], v_scale=[vs]))
        return [x.cpu().numpy() for x in (p, m, ms, v, vs)]


@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("n", [512, 2048, 2048 + 300])
def test_an_overflowing_quotient_is_an_infinity(n, sign):
    """A first moment far above its root and eps: m / (root + eps) leaves binary32, and p becomes an infinity
    of the other sign, as by the division, in whole blocks and in others."""
    eps, at = 1e-10, [5, n - 200, n - 1]
    b = Block8(n)
    for k in {i // 256 for i in at}:
        b.cm[256 * k:256 * (k + 1)], b.ms[k] = 0, np.float32(2.0 ** 100)
    for i in at:
        b.cm[i] = 0x7E if sign > 0 else 0xFE       # 448 of the scale
        b.cv[i], b.g[i] = 0, 0
    m, r, want = b.wanted(7, eps)
    assert np.isinf(want[at]).all() and np.isfinite(np.delete(want, at)).all()
    p, cm, ms, cv, vs = b.step(7, eps)
    assert p[at].tolist() == [-sign * np.inf] * len(at)
    assert np.isfinite(np.delete(p, at)).all()
    for codes, scales, x, roots in ((cm, ms, m, False), (cv, vs, r, True)):
        c, s = R.encode32(x, roots)
        assert np.array_equal(codes, c) and np.array_equal(scales, s)


@pytest.mark.parametrize("state", ["m", "v"])
def test_a_nan_code_makes_its_block_s_scale_nan(state):
    """A NaN among the codes that a caller brings (0x7F, 0xFF) under a finite scale: p is NaN in that element,
    the scale of that state's block becomes NaN, and nothing else differs, in whole blocks and in others."""
    for code in (0x7F, 0xFF):
        for at in (100, 300, 511, 700, 999):            # of 1000 elements the first 512 are two whole blocks
            b = Block8(1000)
            m, r, want = b.wanted(3, 1e-8)
            p0, cm0, ms0, cv0, vs0 = b.step(3, 1e-8)
            (b.cm if state == "m" else b.cv)[at] = code
            p, cm, ms, cv, vs = b.step(3, 1e-8)
            assert np.flatnonzero(np.isnan(p)).tolist() == [at]
            # one form's root and quotient are a unit in the last place off at most, 2^-22 of what p moves by; then
            # p's roundings
            bound = 2.0 ** -22 * np.abs(p0 - b.p) + 2.0 ** -22 * np.maximum(np.abs(p0), np.abs(b.p))
            assert (np.delete(np.abs(p - p0) - bound, at) <= 0).all()
            odd, other = (ms, vs) if state == "m" else (vs, ms)
            assert np.flatnonzero(np.isnan(odd)).tolist() == [at // 256], (code, at)
            assert np.array_equal(other, vs0 if state == "m" else ms0)
            rest = np.arange(1000) // 256 != at // 256
            assert np.array_equal(cm[rest], cm0[rest]) and np.array_equal(cv[rest], cv0[rest])
            assert np.array_equal(odd[~np.isnan(odd)], (ms0 if state == "m" else vs0)[~np.isnan(odd)])


@pytest.mark.parametrize("t", [1, 7, 1000])
def test_parameters_and_roots_of_whole_blocks(t):
    """p and the roots behind the kept scales against each operation in binary32: the same bits where a block
    is ragged, and in whole blocks within one unit in the last place of the root and one of the quotient."""
    n, eps = (1 << 20) + 300, 1e-8
    b = Block8(n, seed=t)
    m, r, want = b.wanted(t, eps)
    p, cm, ms, cv, vs = b.step(t, eps)
    assert np.array_equal(p[1 << 20:], want[1 << 20:])
    # the root's unit, and a product and a sum that may round the other way: 2^-21 of the denominator; the
    # quotient's own; then a product and a difference: 2^-20 of the move and 2^-22 of p
    bound = 2.0 ** -20 * np.abs(want.astype(np.float64) - b.p) + 2.0 ** -22 * np.maximum(np.abs(want), np.abs(b.p))
    off = np.abs(p.astype(np.float64) - want)
    assert (off <= bound).all(), float((off / bound).max())
    assert (p != want).sum() <= 100                 # of a million; one in a million is what the kernel's comment says
    codes, scales = R.encode32(m, False)
    assert np.array_equal(cm, codes) and np.array_equal(ms, scales)
    codes, scales = R.encode32(r, True)
    assert (np.abs(vs.astype(np.float64) - scales) <= 2.0 ** -22 * scales).all()
    assert (cv != codes).sum() <= 20                # a root next to the border between two codes


@pytest.mark.parametrize("t", [1, 7, 1000])
def test_32_bit_states_have_each_operation_s_bits(t):
    b = Block8(5003, seed=t)
    m0, v0 = b.values(b.cm, b.ms), b.values(b.cv, b.vs) ** 2
    m, r, _, want = R.adamw32(b.p, b.g, m0, v0, t, eps=1e-8, wd=0.1, **HYPER)
    p, g, mg, vg = (torch.from_numpy(x.copy()).cuda() for x in (b.p, b.g, m0, v0))
    E.ea_adamw_step(E.AdamW(eps=1e-8, state_bits=32, **HYPER), t, E.TensorList([g], p=[p], m=[mg], v=[vg], weight_decay=0.1))
    assert np.array_equal(mg.cpu().numpy(), m) and np.array_equal(np.sqrt(vg.cpu().numpy()), r)
    assert np.array_equal(p.cpu().numpy(), want)


@pytest.mark.parametrize("kind,master", [("bf16", True), ("bf16", False), ("f32", False)])
def test_long_calls_step_as_short_ones(kind, master):
    """From 2^25 elements on a wave takes four groups of blocks, each fetched while the last is worked on.  The
    same elements in calls of fewer, one group a wave, leave the same bits: values that send a group in the
    middle of a run to the general form (NaN, subnormal second moments, a NaN code) among them."""
    param = {"bf16": torch.bfloat16, "f32": torch.float32}[kind]
    n, cut = (1 << 25) + 5 * 512 + 77, (1 << 24)
    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda scale: torch.randn(n, device="cuda", generator=gen) * scale  # noqa: E731
    w, g = rand(0.1), rand(1e-2)
    m, v = (torch.randint(0, 127, (n,), device="cuda", generator=gen, dtype=torch.uint8) for _ in range(2))
    m |= torch.randint(0, 2, (n,), device="cuda", generator=gen, dtype=torch.uint8) << 7
    ms, vs = (torch.rand(-(-n // 256), device="cuda", generator=gen) * 1e-5 + 1e-6 for _ in range(2))
    # one group of the four of a run for each fault, first to last, in different runs
    for run, (group, fault) in enumerate([(0, "nan"), (1, "small"), (2, "code"), (3, "nan"), (1, "nan"), (2, "small")]):
        at = (1 << 20) + run * 2048 + group * 512 + 100 + run
        if fault == "nan":
            g[at] = float("nan")
        elif fault == "small":
            g[at], v[at], vs[at // 256] = 0, 1, 2.0 ** -55      # its root squares to 2^-128, a subnormal
        else:
            m[at] = 0x7F
    p = w.to(param)
    g = g.to(param)
    outs = []
    for cuts in ([(0, n)], [(0, cut), (cut, n)]):
        got = [x.clone() for x in (p, m, v, ms, vs)] + ([w.clone()] if master else [])
        for a, b in cuts:
            part = [x[a:b] if x.numel() == n else x[a // 256:-(-b // 256)] for x in got]
            tl = E.TensorList([g[a:b]], p=[part[0]], m=[part[1]], v=[part[2]], m_scale=[part[3]], v_scale=[part[4]],
                              master=[part[5]] if master else None, weight_decay=0.01)
            E.ea_adamw_step(E.AdamW(eps=1e-8, state_bits=8, param_type=E.ea_type(param), grad_type=E.ea_type(param),
                                    **HYPER), 5, tl)
        outs.append(got)
    for x, y in zip(*outs):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # the faults reached the blocks they stand in, and no other
    odd = torch.isnan(outs[0][3]).nonzero().view(-1).tolist()
    first = (1 << 20) // 256
    assert odd == [first + 0, first + 8 + 8 + 4 + 0, first + 24 + 6, first + 32 + 2], odd
    # each block against the formula, around the faults and at the ends
    m32 = lambda c, s, a, b: R.VALUES[c[a:b].cpu().numpy()].astype(np.float32) * \
        np.repeat(s[a // 256:-(-b // 256)].cpu().numpy(), 256)[:b - a]  # noqa: E731
    for a, b in ((0, 2048), ((1 << 20) - 2048, (1 << 20) + 8 * 2048), ((1 << 25) - 2048, n)):
        with np.errstate(invalid="ignore"):
            r0 = m32(v, vs, a, b)
            start = (w if master else p)[a:b].float().cpu().numpy()
            mk, rk, _, pk = R.adamw32(start, g[a:b].float().cpu().numpy(), m32(m, ms, a, b), r0 * r0, 5, eps=1e-8, wd=0.01,
                                      **HYPER)
        fine = ~np.repeat(np.isnan(R.pad(mk)).any(1) | np.isnan(R.pad(rk)).any(1), 256)[:b - a]
        for codes, scales, x, roots in ((1, 3, mk, False), (2, 4, rk, True)):
            want, s = R.encode32(np.where(fine, x, 0), roots)
            got = outs[0][codes][a:b].cpu().numpy()
            assert (got[fine] != want[fine]).sum() <= (2 if roots else 0)      # a root next to the border of two codes
        got = outs[0][5 if master else 0][a:b].float().cpu().numpy()
        bound = 2.0 ** -20 * np.abs(pk - start) + 2.0 ** -22 * np.maximum(np.abs(pk), np.abs(start))
        if not master and kind == "bf16":
            bound = bound + 2.0 ** -8 * np.abs(pk)
        odd = np.isnan(pk)
        assert np.array_equal(np.isnan(got), odd) and (np.abs(got - pk)[~odd] <= bound[~odd]).all()
