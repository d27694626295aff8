"""Host-side checks of the layers' operators (no GPU work): the header's symbols and structures, sizes, and calls that
are refused before any device work."""
import ctypes as C
import math
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "ea_layer.h")
P = 1 << 20                                       # stands for device memory; a refused call does not touch it
ARG, ALIGN, UNSUPPORTED = -1, -2, -4


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
    assert names == ["ea_dropout", "ea_dropout_grad", "ea_layer_norm", "ea_layer_norm_grad", "ea_layer_norm_workspace_bytes",
                     "ea_recurrence", "ea_recurrence_grad", "ea_recurrence_states_bytes", "ea_recurrence_workspace_bytes",
                     "ea_token_loss", "ea_token_loss_workspace_bytes"]
    for n in names:
        assert hasattr(E.lib, n) and callable(getattr(E, n)), n
        assert n in E.__all__
    for n, v in re.findall(r"#define (EA_[A-Z_]+) +(\d+)", open(HEADER).read()):
        assert getattr(E, n) == int(v)


def test_structures_have_the_header_s_layout(E, tmp_path):
    classes = ((E.LayerNorm, "ea_layer_norm_t"), (E.Dropout, "ea_dropout_t"), (E.Recurrence, "ea_recurrence_t"),
               (E.TokenLoss, "ea_token_loss_t"))
    lines = []
    for cls, name in classes:
        lines.append(f'printf("%zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {f}));' for f, _ in cls._fields_] + ['printf("\\n");']
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "ea_layer.h"\nint main(void) {' + "\n".join(lines) +
                   "return 0; }\n")
    exe = str(tmp_path / "layout")
    env = {k: v for k, v in os.environ.items() if k != "LD_PRELOAD"}
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.dirname(HEADER), str(src), "-o", exe], check=True,
                   env=env)
    got = subprocess.run([exe], capture_output=True, text=True, check=True, env=env).stdout.splitlines()
    for line, (cls, _) in zip(got, classes):
        assert [int(x) for x in line.split()] == [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_]


class Op:
    """An entry point with arguments it would take, all but the stream by name; `call` with some of them replaced."""

    def __init__(self, fn, config, **args):
        self.fn, self.config, self.args = fn, config, args

    def call(self, config=None, **kw):
        a = {**self.args, **kw}
        return self.fn(None if config is False else C.byref(config or self.config()), *a.values(), None)


def norm_config(E, **kw):
    return E.LayerNorm(**{**dict(rows=4, dim=6, x_stride=6, y_stride=6, eps=1e-5), **kw})


def drop_config(E, **kw):
    return E.Dropout(**{**dict(rows=4, dim=6, x_stride=6, y_stride=6, p=0.1), **kw})


def rec_config(E, **kw):
    return E.Recurrence(**{**dict(batch=2, length=3, dim=6, x_stride=6, g_stride=6, y_stride=6, gate=1), **kw})


def loss_config(E, **kw):
    return E.TokenLoss(**{**dict(rows=4, vocab=6, logits_stride=6, dlogits_stride=6, scale=1.0, index_bits=64), **kw})


def operators(E):
    L = E.lib
    norm, drop = lambda: norm_config(E), lambda: drop_config(E)  # noqa: E731
    rec, loss = lambda: rec_config(E), lambda: loss_config(E)  # noqa: E731
    return {
        "norm": Op(L.ea_layer_norm, norm, x=P, weight=P, bias=P, y=2 * P, mean=P, rstd=P),
        "norm_grad": Op(L.ea_layer_norm_grad, norm, x=P, dy=P, weight=P, mean=P, rstd=P, add=P, dx=2 * P, dweight=P,
                        dbias=P, accumulate=0, workspace=P),
        "drop": Op(L.ea_dropout, drop, t=1, t_dev=None, x=P, residual=P, y=2 * P),
        "drop_grad": Op(L.ea_dropout_grad, drop, t=1, t_dev=None, dy=P, dx=2 * P),
        "rec": Op(L.ea_recurrence, rec, g=P, x=P, h0=P, lengths=P, y=P, states=P, h_last=P, workspace=P),
        "rec_grad": Op(L.ea_recurrence_grad, rec, g=P, x=P, states=P, lengths=P, dy=P, dh_last=P, dg=P, dx=P, dh0=P,
                       workspace=P),
        "loss": Op(L.ea_token_loss, loss, logits=P, targets=P, loss=P, total=P, count=P, dlogits=2 * P, workspace=P),
    }


BAD_CONFIGS = {
    "norm": [dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=-3), dict(dim=(1 << 20) + 1, x_stride=1 << 21, y_stride=1 << 21),
             dict(x_stride=5), dict(y_stride=5), dict(x_stride=1 << 32), dict(y_stride=1 << 32), dict(eps=0.0), dict(eps=-1.0),
             dict(eps=math.nan), dict(eps=math.inf), dict(x_type=3), dict(y_type=-1), dict(w_type=7)],
    "drop": [dict(rows=-1), dict(rows=1 << 31), dict(dim=0), dict(dim=(1 << 30) + 1, x_stride=1 << 31, y_stride=1 << 31),
             dict(x_stride=5), dict(y_stride=5), dict(x_stride=1 << 32), dict(y_stride=1 << 32), dict(p=-0.1), dict(p=1.1),
             dict(p=math.nan), dict(p=math.inf), dict(x_type=3), dict(y_type=-1)],
    "rec": [dict(batch=-1), dict(batch=1 << 31), dict(length=-1), dict(length=1 << 31), dict(dim=0),
            dict(dim=(1 << 20) + 1, x_stride=1 << 21, g_stride=1 << 21, y_stride=1 << 21), dict(x_stride=5), dict(g_stride=5),
            dict(y_stride=5), dict(x_stride=1 << 32), dict(g_stride=1 << 32), dict(y_stride=1 << 32), dict(gate=2), dict(gate=-1),
            dict(x_type=3), dict(g_type=-1), dict(reserved=1)],
    "loss": [dict(rows=-1), dict(rows=1 << 31), dict(vocab=0), dict(vocab=(1 << 24) + 1, logits_stride=1 << 25, dlogits_stride=1 << 25),
             dict(logits_stride=5), dict(dlogits_stride=5), dict(logits_stride=1 << 32), dict(dlogits_stride=1 << 32),
             dict(scale=math.nan), dict(scale=math.inf), dict(type=3), dict(index_bits=16), dict(index_bits=0), dict(reduction=2),
             dict(reduction=-1)],
}
MAKE = dict(norm=norm_config, drop=drop_config, rec=rec_config, loss=loss_config)
SIZES = dict(norm=["ea_layer_norm_workspace_bytes"], drop=[], rec=["ea_recurrence_workspace_bytes", "ea_recurrence_states_bytes"],
             loss=["ea_token_loss_workspace_bytes"])


@pytest.mark.parametrize("kind,bad", [(k, b) for k, v in BAD_CONFIGS.items() for b in v], ids=str)
def test_configurations_are_refused(E, kind, bad):
    c = MAKE[kind](E, **bad)
    for name, op in operators(E).items():
        if name.split("_")[0] == kind:
            assert op.call(c) == ARG and E.ea_last_error(), name
    for size in SIZES[kind]:
        assert getattr(E.lib, size)(C.byref(c)) == ARG
        with pytest.raises(E.EAError):
            getattr(E, size)(c)


def test_no_configuration_is_refused(E):
    for op in operators(E).values():
        assert op.call(False) == ARG
    for names in SIZES.values():
        for size in names:
            assert getattr(E.lib, size)(None) == ARG


REQUIRED = dict(norm=["x", "y"], norm_grad=["x", "dy", "mean", "rstd", "dx", "workspace"], drop=["x", "y"], drop_grad=["dy", "dx"],
                rec=["g", "x", "y"], rec_grad=["g", "x", "states", "dy", "dg", "dx"],
                loss=["logits", "targets", "total", "workspace"])


@pytest.mark.parametrize("name", REQUIRED)
def test_missing_and_misaligned_pointers_are_refused(E, name):
    op = operators(E)[name]
    for arg in REQUIRED[name]:
        assert op.call(**{arg: None}) == ARG and arg in E.ea_last_error(), arg
    for arg in op.args:
        if arg in ("t", "accumulate") or (arg == "workspace" and name.startswith("rec")):
            continue
        assert op.call(**{arg: P + 1}) == ALIGN and arg in E.ea_last_error(), arg


def test_arguments_are_refused(E):
    ops = operators(E)
    for t in (-1, 1 << 32):
        assert ops["drop"].call(t=t) == ARG and ops["drop_grad"].call(t=t) == ARG
    assert ops["drop"].call(t_dev=P + 2) == ALIGN
    assert ops["norm_grad"].call(accumulate=2) == ARG and ops["norm_grad"].call(accumulate=-1) == ARG
    assert ops["norm_grad"].call(workspace=P + 8) == ALIGN and ops["loss"].call(workspace=P + 8) == ALIGN
    long = rec_config(E, batch=1, length=5000)
    assert ops["rec"].call(long, workspace=None) == ARG and ops["rec_grad"].call(long, workspace=P + 8) == ALIGN
    assert ops["rec"].call(rec_config(E, batch=1 << 16, length=1 << 15)) == UNSUPPORTED
    wide = dict(dim=1 << 20, x_stride=1 << 20, g_stride=1 << 20, y_stride=1 << 20)
    large = rec_config(E, batch=1 << 10, length=1 << 20, **wide)
    assert ops["rec"].call(large) == UNSUPPORTED and ops["rec_grad"].call(large) == UNSUPPORTED
    # one array in two roles needs one type and stride
    for name, out, kw in (("norm", "y", dict(y_type=E.EA_BF16)), ("norm", "y", dict(y_stride=8)),
                          ("drop", "y", dict(y_type=E.EA_BF16)), ("drop", "y", dict(x_stride=8)),
                          ("drop_grad", "dx", dict(x_type=E.EA_F16)), ("drop_grad", "dx", dict(x_stride=8)),
                          ("norm_grad", "dx", dict(y_type=E.EA_BF16)), ("norm_grad", "dx", dict(y_stride=8)),
                          ("loss", "dlogits", dict(dlogits_stride=8))):
        kind = name.split("_")[0]
        assert ops[name].call(MAKE[kind](E, **kw), **{out: P}) == ARG, (name, kw)
        assert "one array" in E.ea_last_error()


def test_nothing_to_do_needs_no_arrays(E):
    ops = operators(E)
    none = {n: {a: None for a in op.args if a not in ("t", "accumulate", "total")} for n, op in ops.items()}
    assert ops["norm"].call(norm_config(E, rows=0), **none["norm"]) == 0
    assert ops["norm_grad"].call(norm_config(E, rows=0), **none["norm_grad"]) == 0
    assert ops["drop"].call(drop_config(E, rows=0), **none["drop"]) == 0
    assert ops["drop_grad"].call(drop_config(E, rows=0), **none["drop_grad"]) == 0
    assert ops["rec"].call(rec_config(E, batch=0), **none["rec"]) == 0
    assert ops["rec_grad"].call(rec_config(E, batch=0), **none["rec_grad"]) == 0


def test_sizes(E):
    for rows, dim in ((1, 1), (10, 768), (10 ** 6, 4096), (2 ** 31 - 1, 2 ** 20)):
        n = E.ea_layer_norm_workspace_bytes(norm_config(E, rows=rows, dim=dim, x_stride=dim, y_stride=dim))
        assert 0 < n <= 8 * -(-dim // 8) * 8 * min(rows, 4096)
    for b, n, dim in ((1, 1, 1), (3, 64, 5), (3, 65, 5), (1, 65_536, 1024), (2 ** 10, 2 ** 10, 2 ** 20)):
        c = rec_config(E, batch=b, length=n, dim=dim, x_stride=dim, g_stride=dim, y_stride=dim)
        assert E.ea_recurrence_states_bytes(c) == 4 * b * -(-n // 64) * dim
        # a product and an end value for every 128 steps and every group of 16 such, of 8 bytes each, and a state for
        # every stretch of groups
        chunks = -(-n // 128)
        assert 0 <= E.ea_recurrence_workspace_bytes(c) <= 8 * (16 + b * dim * (2 * chunks + 2 * -(-chunks // 16) + chunks))
    for rows, vocab in ((1, 1), (2048, 32_000), (2 ** 31 - 1, 2 ** 24)):
        n = E.ea_token_loss_workspace_bytes(loss_config(E, rows=rows, vocab=vocab, logits_stride=vocab, dlogits_stride=vocab))
        # the waves' sums; rows that are not held: 16 bytes and a logit each, and 8 bytes for a piece of 8,192 logits
        held = 16 * (9000 + 256)
        assert 0 < n <= (held if vocab <= 65_000 else held + rows * (20 + 8 * (vocab // 8192 + 2)))


def test_host_tensors_and_wrong_ones_are_refused(E):
    torch = pytest.importorskip("torch")
    x, w, i = torch.zeros(4, 6), torch.zeros(6), torch.zeros(4, dtype=torch.int64)
    calls = (lambda: E.ea_layer_norm(norm_config(E), x, w, w, x, stream=0),
             lambda: E.ea_layer_norm_grad(norm_config(E), x, x, w, i, i, None, x, w, w, False, None, stream=0),
             lambda: E.ea_dropout(drop_config(E), 1, x, None, x, stream=0),
             lambda: E.ea_dropout_grad(drop_config(E), 1, x, x, stream=0),
             lambda: E.ea_recurrence(rec_config(E), x, x, None, None, x, None, None, None, stream=0),
             lambda: E.ea_recurrence_grad(rec_config(E), x, x, w, None, x, None, x, x, None, None, stream=0),
             lambda: E.ea_token_loss(loss_config(E), x, i, None, w, None, None, None, stream=0))
    for call in calls:
        with pytest.raises(ValueError, match="device tensors"):
            call()
    for bad in (dict(x_type=9), dict(x_type=-1)):
        with pytest.raises(ValueError, match="x_type"):
            E.ea_layer_norm(norm_config(E, **bad), x, w, w, x, stream=0)
    with pytest.raises(ValueError, match="index_bits"):
        E.ea_token_loss(loss_config(E, index_bits=8), x, i, None, w, None, None, None, stream=0)
