"""Host-side checks of the operators beside the round (no GPU work): the header's symbols and
structures, sizes, and calls that are refused before any device work."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ea_train.h")
P = 1 << 20                                       # stands for device memory; a refused call does not touch it


@pytest.fixture(scope="module")
def E():
    from paper_2205_14473_amd import build as bld
    if bld.is_stale() and "EA_LIB" not in os.environ:
        bld.build()
    import paper_2205_14473_amd as E
    return E


def test_every_declared_symbol_is_exported_and_bound(E):
    src = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = sorted(set(re.findall(r"\b(ea_[a-z_0-9]+)\s*\(", src)))
    assert names == ["ea_adamw_step", "ea_adamw_step_scheduled", "ea_embed_grad", "ea_embed_lookup",
                     "ea_embed_workspace_bytes", "ea_grad_norm", "ea_grad_norm_workspace_bytes"]
    for n in names:
        assert hasattr(E.lib, n) and callable(getattr(E, n)), n


def test_structures_have_the_header_s_layout(E, tmp_path):
    lines = []
    for cls, name in ((E.Tensor, "ea_tensor_t"), (E.AdamW, "ea_adamw_t"), (E.Embed, "ea_embed_t")):
        lines.append(f'printf("%zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {f}));' for f, _ in cls._fields_] + ['printf("\\n");']
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ea_train.h"\nint main(void) {' + "\n".join(lines) +
                   "return 0; }\n")
    exe = str(tmp_path / "layout")
    env = {k: v for k, v in os.environ.items() if k != "LD_PRELOAD"}
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), str(src), "-o", exe], check=True,
                   env=env)
    got = subprocess.run([exe], capture_output=True, text=True, check=True, env=env).stdout.splitlines()
    for line, cls in zip(got, (E.Tensor, E.AdamW, E.Embed)):
        assert [int(x) for x in line.split()] == [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]


def adamw(E, **kw):
    return E.AdamW(**{**dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, state_bits=32), **kw})


def tensor(E, **kw):
    return E.Tensor(**{**dict(g=P, p=P, m=P, v=P, m_scale=P, v_scale=P, n=8, lr_scale=1.0), **kw})


def step(E, cfg, ts, t=1, gscale=None):
    array = (E.Tensor * max(1, len(ts)))(*ts)
    return E.lib.ea_adamw_step(C.byref(cfg) if cfg is not None else None, t, len(ts), array, gscale, None)


BAD_CONFIGS = [dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(beta1=1.0), dict(beta1=-0.1),
               dict(beta1=math.nan), dict(beta2=1.0), dict(beta2=math.nan), dict(eps=0.0), dict(eps=-1.0),
               dict(eps=math.inf), dict(param_type=3), dict(grad_type=-1), dict(state_bits=16), dict(state_bits=0),
               dict(rounding=2, state_bits=8), dict(rounding=1)]


@pytest.mark.parametrize("bad", BAD_CONFIGS, ids=str)
def test_step_refuses_configurations(E, bad):
    assert step(E, adamw(E, **bad), [tensor(E)]) == E.EA_ERR_ARG
    assert E.ea_last_error()


BAD_TENSORS = [(dict(n=-1), -1), (dict(n=1 << 40), -1), (dict(g=None), -1), (dict(p=None), -1), (dict(m=None), -1),
               (dict(v=None), -1), (dict(g=P + 2), -2), (dict(p=P + 1), -2), (dict(m=P + 2), -2), (dict(v=P + 3), -2),
               (dict(weight_decay=-0.1), -1), (dict(weight_decay=math.nan), -1), (dict(lr_scale=-1.0), -1),
               (dict(lr_scale=math.inf), -1), (dict(master=P), -1)]


@pytest.mark.parametrize("bad,code", BAD_TENSORS, ids=str)
def test_step_refuses_tensors(E, bad, code):
    assert step(E, adamw(E), [tensor(E), tensor(E, **bad)]) == code
    assert "tensor 1" in E.ea_last_error()


def test_step_refuses_8_bit_states_without_scales_and_bad_alignment(E):
    cfg = adamw(E, state_bits=8, param_type=E.EA_BF16)
    for bad, code in ((dict(m_scale=None), -1), (dict(v_scale=None), -1), (dict(m_scale=P + 2), -2),
                      (dict(p=P + 1), -2), (dict(master=P + 2), -2)):
        assert step(E, cfg, [tensor(E, **bad)]) == code, bad
    assert step(E, adamw(E), [tensor(E)], gscale=P + 1) == E.EA_ERR_ALIGN


def test_step_refuses_lists_and_steps(E):
    assert step(E, None, [tensor(E)]) == E.EA_ERR_ARG
    for t in (0, -1, 1 << 32):
        assert step(E, adamw(E), [tensor(E)], t=t) == E.EA_ERR_ARG
    f = E.lib.ea_adamw_step
    assert f(C.byref(adamw(E)), 1, -1, None, None, None) == E.EA_ERR_ARG
    assert f(C.byref(adamw(E)), 1, 1, None, None, None) == E.EA_ERR_ARG
    assert step(E, adamw(E), [tensor(E, n=(1 << 40) - 1), tensor(E, n=2)]) == E.EA_ERR_UNSUPPORTED
    # nothing to do is no error, and no device work
    assert step(E, adamw(E), []) == 0
    assert step(E, adamw(E), [tensor(E, n=0, g=None, p=None, m=None, v=None)]) == 0


def test_scheduled_step_refuses_schedules(E):
    f = E.lib.ea_adamw_step_scheduled
    ts = (E.Tensor * 1)(tensor(E))

    def call(s, t_dev=P):
        return f(C.byref(adamw(E)), C.byref(s) if s is not None else None, t_dev, 1, ts, None, None)

    assert call(None) == E.EA_ERR_ARG
    assert call(E.Schedule(kind=9)) == E.EA_ERR_ARG
    assert call(E.Schedule(kind=E.EA_SCHED_ASSUMPTION2, alpha=1.0, theta=2.0, T=1)) == E.EA_ERR_ARG
    assert call(E.Schedule(kind=E.EA_SCHED_ASSUMPTION2, alpha=1.0, theta=1e-9, T=1 << 20)) == E.EA_ERR_ARG
    assert call(E.Schedule(), None) == E.EA_ERR_ALIGN and call(E.Schedule(), P + 2) == E.EA_ERR_ALIGN
    ts[0].p = None
    assert call(E.Schedule()) == E.EA_ERR_ARG


def norm(E, ts, kind=0, scale=1.0, most=1.0, out=P, factor=P, ws=P):
    array = (E.Tensor * max(1, len(ts)))(*ts)
    return E.lib.ea_grad_norm(kind, len(ts), array, scale, most, out, factor, ws, None)


def test_norm_refuses(E):
    ts = [tensor(E)]
    assert norm(E, ts, kind=7) == E.EA_ERR_ARG
    for scale in (0.0, -1.0, math.nan, math.inf):
        assert norm(E, ts, scale=scale) == E.EA_ERR_ARG
    for most in (0.0, -1.0, math.nan):
        assert norm(E, ts, most=most) == E.EA_ERR_ARG
    assert norm(E, ts, out=None) == E.EA_ERR_ARG and norm(E, ts, out=P + 1) == E.EA_ERR_ALIGN
    assert norm(E, ts, factor=P + 2) == E.EA_ERR_ALIGN
    assert norm(E, ts, ws=None) == E.EA_ERR_ARG and norm(E, ts, ws=P + 4) == E.EA_ERR_ALIGN
    assert norm(E, [tensor(E, g=None)]) == E.EA_ERR_ARG and norm(E, [tensor(E, g=P + 1)]) == E.EA_ERR_ALIGN
    assert norm(E, [tensor(E, g=P + 1)], kind=E.EA_BF16) == E.EA_ERR_ALIGN
    assert norm(E, [tensor(E, n=-5)]) == E.EA_ERR_ARG


def test_norm_workspace(E):
    size = lambda ts: E.lib.ea_grad_norm_workspace_bytes(len(ts), (E.Tensor * max(1, len(ts)))(*ts))  # noqa: E731
    assert size([]) == 0 and size([tensor(E, n=0)]) == 0
    assert size([tensor(E, n=-1)]) < 0
    for n in (1, 4096, 4097, 10 ** 6, 10 ** 9, 10 ** 11):
        assert 8 <= size([tensor(E, n=n)]) <= 8 * 8200 and size([tensor(E, n=n)]) % 8 == 0
    assert size([tensor(E, n=1)] * 300) == 8 * 300


def embed(E, **kw):
    return E.Embed(**{**dict(tokens=10, vocab=7, dim=6, table_stride=6, x_stride=6, padding=-1, scale=1.0,
                             index_bits=64), **kw})


BAD_EMBEDS = [dict(tokens=-1), dict(tokens=1 << 30), dict(vocab=0), dict(vocab=(1 << 31) - 1), dict(dim=0),
              dict(dim=(1 << 20) + 1, table_stride=1 << 21, x_stride=1 << 21), dict(table_stride=5), dict(x_stride=5),
              dict(table_stride=1 << 32), dict(x_stride=1 << 32), dict(scale=math.nan), dict(scale=math.inf),
              dict(table_type=3), dict(x_type=-1), dict(index_bits=16)]


@pytest.mark.parametrize("bad", BAD_EMBEDS, ids=str)
def test_embedding_refuses_configurations(E, bad):
    c = C.byref(embed(E, **bad))
    assert E.lib.ea_embed_lookup(c, P, P, P, None) == E.EA_ERR_ARG
    assert E.lib.ea_embed_grad(c, P, P, P, 0, P, None) == E.EA_ERR_ARG
    assert E.lib.ea_embed_workspace_bytes(c) == E.EA_ERR_ARG


def test_embedding_refuses_pointers(E):
    c = C.byref(embed(E))
    for bad, code in ((None, E.EA_ERR_ARG), (P + 2, E.EA_ERR_ALIGN)):
        for k in range(3):
            a = [P, P, P]
            a[k] = bad
            assert E.lib.ea_embed_lookup(c, *a, None) == code
            assert E.lib.ea_embed_grad(c, *a, 0, P, None) == code
    assert E.lib.ea_embed_grad(c, P, P, P, 0, None, None) == E.EA_ERR_ARG
    assert E.lib.ea_embed_grad(c, P, P, P, 0, P + 8, None) == E.EA_ERR_ALIGN
    assert E.lib.ea_embed_grad(c, P, P, P, 2, P, None) == E.EA_ERR_ARG
    assert E.lib.ea_embed_lookup(None, P, P, P, None) == E.EA_ERR_ARG
    assert E.lib.ea_embed_lookup(C.byref(embed(E, tokens=0)), None, None, None, None) == 0
    assert E.lib.ea_embed_grad(C.byref(embed(E, tokens=0)), None, None, P, 1, None, None) == 0
    assert E.lib.ea_embed_workspace_bytes(C.byref(embed(E, tokens=0))) == 0


def test_embedding_workspace_grows_with_the_tokens(E):
    last = 0
    for n in (1, 100, 4096, 4097, 300_000, 10 ** 7, (1 << 30) - 1):
        size = E.ea_embed_workspace_bytes(embed(E, tokens=n, dim=1024, table_stride=1024, x_stride=1024, vocab=50_000))
        assert size > last and size <= n * 16 + 64 * 4096 + (n // 2 + 64) * 1024 * 4 * 2
        last = size


def test_host_tensors_are_refused(E):
    torch = pytest.importorskip("torch")
    t = torch.zeros(8)
    with pytest.raises(ValueError, match="device tensors"):
        E.TensorList([t], p=[t], m=[t], v=[t])
    with pytest.raises(ValueError, match="device tensors"):
        E.TensorList([t])
    with pytest.raises(ValueError, match="device tensors"):
        E.ea_embed_lookup(embed(E), torch.zeros(7, 6), torch.zeros(10, dtype=torch.int64), torch.zeros(10, 6), 0)
    for bad in (None, 3):
        with pytest.raises(ValueError, match=r"g\[1\]: expected a tensor|device tensors"):
            E.TensorList([t, bad])
        with pytest.raises(ValueError, match=r"g\[0\]: expected a tensor"):
            E.TensorList([bad, t])
    with pytest.raises(ValueError, match="2 tensors in p, and 1 in g"):
        E.TensorList([t], p=[t, t])
