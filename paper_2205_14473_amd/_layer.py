"""ctypes binding of the layers' operators (include/ea_layer.h): layer norm,
dropout, the gated linear recurrence and the token loss, with their gradients.
Argument marshalling only, in the manner of ``_train``: every function has the
name of the C entry point it calls, tensors are device tensors of the documented
types, on the current device, streams are torch streams, raw hipStream_t
integers, or None for torch's current stream.  A raw pointer (an integer) may
stand for any tensor; nothing is checked of it but its alignment.
"""
import ctypes as C

from . import _binding as B
from . import _train as T
from ._binding import _check, lib

EA_GATE_PLAIN, EA_GATE_SIGMOID = 0, 1
EA_RECURRENCE_BLOCK = 64
EA_REDUCE_MEAN, EA_REDUCE_SUM = 0, 1

_P, _I32, _I64 = C.c_void_p, C.c_int32, C.c_int64


class LayerNorm(C.Structure):
    """ea_layer_norm_t"""
    _fields_ = [("rows", _I64), ("dim", _I64), ("x_stride", _I64), ("y_stride", _I64), ("eps", C.c_float),
                ("x_type", _I32), ("y_type", _I32), ("w_type", _I32)]


class Dropout(C.Structure):
    """ea_dropout_t"""
    _fields_ = [("rows", _I64), ("dim", _I64), ("x_stride", _I64), ("y_stride", _I64), ("p", C.c_float),
                ("x_type", _I32), ("y_type", _I32), ("site", C.c_uint32), ("seed", C.c_uint64)]


class Recurrence(C.Structure):
    """ea_recurrence_t"""
    _fields_ = [("batch", _I64), ("length", _I64), ("dim", _I64), ("x_stride", _I64), ("g_stride", _I64),
                ("y_stride", _I64), ("gate", _I32), ("x_type", _I32), ("g_type", _I32), ("reserved", _I32)]


class TokenLoss(C.Structure):
    """ea_token_loss_t"""
    _fields_ = [("rows", _I64), ("vocab", _I64), ("logits_stride", _I64), ("dlogits_stride", _I64),
                ("scale", C.c_float), ("type", _I32), ("index_bits", _I32), ("reduction", _I32)]


assert C.sizeof(LayerNorm) == 48 and C.sizeof(Dropout) == 56
assert C.sizeof(Recurrence) == 64 and C.sizeof(TokenLoss) == 48

for _name, _res, _args in (
        ("ea_layer_norm", C.c_int, [C.POINTER(LayerNorm)] + [_P] * 7),
        ("ea_layer_norm_workspace_bytes", _I64, [C.POINTER(LayerNorm)]),
        ("ea_layer_norm_grad", C.c_int, [C.POINTER(LayerNorm)] + [_P] * 9 + [_I32, _P, _P]),
        ("ea_dropout", C.c_int, [C.POINTER(Dropout), _I64] + [_P] * 5),
        ("ea_dropout_grad", C.c_int, [C.POINTER(Dropout), _I64] + [_P] * 4),
        ("ea_recurrence_states_bytes", _I64, [C.POINTER(Recurrence)]),
        ("ea_recurrence_workspace_bytes", _I64, [C.POINTER(Recurrence)]),
        ("ea_recurrence", C.c_int, [C.POINTER(Recurrence)] + [_P] * 9),
        ("ea_recurrence_grad", C.c_int, [C.POINTER(Recurrence)] + [_P] * 11),
        ("ea_token_loss_workspace_bytes", _I64, [C.POINTER(TokenLoss)]),
        ("ea_token_loss", C.c_int, [C.POINTER(TokenLoss)] + [_P] * 8)):
    getattr(lib, _name).restype, getattr(lib, _name).argtypes = _res, _args


class _Call:
    """The tensors of one call, checked one after the other, and the device they share.  A small call takes the
    GPU 2 to 4 us, so the plain way through each check is short."""
    __slots__ = ("device",)

    def __init__(self):
        self.device = None

    def on(self, t, name):
        d = t.get_device()
        if d != self.device:
            if d < 0:
                raise ValueError("libea needs device tensors")
            if self.device is not None:
                raise ValueError(f"{name} is on {t.device}, and others on device {self.device}")
            self.device = d

    def rows(self, t, kind, rows, dim, stride, name):
        """Pointer of a [rows, dim] tensor (leading dimensions may be split) with `stride` elements between rows."""
        if t is None or t.__class__ is int:
            return t
        self.on(t, name)
        if t.dtype is (T._types or T._dtypes())[kind] and t.shape == (rows, dim) and t.stride() == (stride, 1):
            return t.data_ptr()
        return T._rows(t, kind, rows, dim, stride, name)

    def flat(self, t, dtype, count, name):
        """Pointer of `count` contiguous elements."""
        if t is None or t.__class__ is int:
            return t
        self.on(t, name)
        if t.dtype is not dtype:
            raise ValueError(f"{name}: expected {dtype}, got {t.dtype}")
        if t.numel() != count or not t.is_contiguous():
            raise ValueError(f"{name}: expected {count} contiguous elements, got shape {tuple(t.shape)}, strides "
                             f"{t.stride()}")
        return t.data_ptr()

    def weights(self, t, kind, dim, name):
        return self.flat(t, (T._types or T._dtypes())[kind], dim, name)

    def floats(self, t, count, name):
        return self.flat(t, (T._types or T._dtypes())[T.EA_F32], count, name)

    def workspace(self, t, need):
        if t is None or t.__class__ is int:
            return t
        self.on(t, "workspace")
        T._room(t, need)
        return B._ptr(t)

    def step(self, t_dev):
        if t_dev is None or t_dev.__class__ is int:
            return t_dev
        self.on(t_dev, "t_dev")
        if t_dev.numel() < 1:
            raise ValueError("t_dev: expected one element, got none")
        return B._ptr_u32(t_dev)

    def queue(self, stream):
        return T._queue(stream, self.device)


def _kind(kind, name):
    """An element type of a configuration, before it is looked up."""
    if kind not in (T.EA_F32, T.EA_BF16, T.EA_F16):
        raise ValueError(f"unknown {name} {kind}")
    return kind


def ea_layer_norm(cfg, x, weight, bias, y, mean=None, rstd=None, stream=None):
    c, n, dim = _Call(), cfg.rows, cfg.dim
    xt, yt, wt = _kind(cfg.x_type, "x_type"), _kind(cfg.y_type, "y_type"), _kind(cfg.w_type, "w_type")
    return _check(lib.ea_layer_norm(
        C.byref(cfg), c.rows(x, xt, n, dim, cfg.x_stride, "x"), c.weights(weight, wt, dim, "weight"),
        c.weights(bias, wt, dim, "bias"), c.rows(y, yt, n, dim, cfg.y_stride, "y"), c.floats(mean, n, "mean"),
        c.floats(rstd, n, "rstd"), c.queue(stream)))


def ea_layer_norm_workspace_bytes(cfg) -> int:
    return _check(lib.ea_layer_norm_workspace_bytes(C.byref(cfg)))


def ea_layer_norm_grad(cfg, x, dy, weight, mean, rstd, add, dx, dweight, dbias, accumulate, workspace, stream=None):
    c, n, dim = _Call(), cfg.rows, cfg.dim
    xt, yt, wt = _kind(cfg.x_type, "x_type"), _kind(cfg.y_type, "y_type"), _kind(cfg.w_type, "w_type")
    need = 0 if dweight is None and dbias is None else lib.ea_layer_norm_workspace_bytes(C.byref(cfg))
    return _check(lib.ea_layer_norm_grad(
        C.byref(cfg), c.rows(x, xt, n, dim, cfg.x_stride, "x"), c.rows(dy, yt, n, dim, cfg.y_stride, "dy"),
        c.weights(weight, wt, dim, "weight"), c.floats(mean, n, "mean"), c.floats(rstd, n, "rstd"),
        c.rows(add, xt, n, dim, cfg.x_stride, "add"), c.rows(dx, xt, n, dim, cfg.x_stride, "dx"),
        c.weights(dweight, wt, dim, "dweight"), c.weights(dbias, wt, dim, "dbias"), 1 if accumulate else 0,
        c.workspace(workspace, need), c.queue(stream)))


def ea_dropout(cfg, t, x, residual, y, t_dev=None, stream=None):
    c, n, dim = _Call(), cfg.rows, cfg.dim
    xt, yt = _kind(cfg.x_type, "x_type"), _kind(cfg.y_type, "y_type")
    return _check(lib.ea_dropout(
        C.byref(cfg), t, c.step(t_dev), c.rows(x, xt, n, dim, cfg.x_stride, "x"),
        c.rows(residual, yt, n, dim, cfg.y_stride, "residual"), c.rows(y, yt, n, dim, cfg.y_stride, "y"),
        c.queue(stream)))


def ea_dropout_grad(cfg, t, dy, dx, t_dev=None, stream=None):
    c, n, dim = _Call(), cfg.rows, cfg.dim
    xt, yt = _kind(cfg.x_type, "x_type"), _kind(cfg.y_type, "y_type")
    return _check(lib.ea_dropout_grad(
        C.byref(cfg), t, c.step(t_dev), c.rows(dy, yt, n, dim, cfg.y_stride, "dy"),
        c.rows(dx, xt, n, dim, cfg.x_stride, "dx"), c.queue(stream)))


def ea_recurrence_states_bytes(cfg) -> int:
    return _check(lib.ea_recurrence_states_bytes(C.byref(cfg)))


def ea_recurrence_workspace_bytes(cfg) -> int:
    return _check(lib.ea_recurrence_workspace_bytes(C.byref(cfg)))


class _Sequences(_Call):
    """Arrays of [batch, length, dim], [batch, blocks, dim] and [batch, dim]."""
    __slots__ = ("cfg",)

    def __init__(self, cfg):
        super().__init__()
        self.cfg = cfg

    def steps(self, t, kind, stride, name):
        if t is None or t.__class__ is int:
            return t
        self.on(t, name)
        b, n, dim = self.cfg.batch, self.cfg.length, self.cfg.dim
        if t.dtype is (T._types or T._dtypes())[kind] and t.shape == (b, n, dim) and \
                t.stride() == (n * stride, stride, 1):
            return t.data_ptr()
        return T._rows(t, kind, b * n, dim, stride, name)

    def ends(self, t, name):
        return self.floats(t, self.cfg.batch * self.cfg.dim, name)

    def states(self, t):
        blocks = (self.cfg.length + EA_RECURRENCE_BLOCK - 1) // EA_RECURRENCE_BLOCK
        return self.floats(t, self.cfg.batch * blocks * self.cfg.dim, "states")

    def lengths(self, t):
        if t is None or t.__class__ is int:
            return t
        T._dtypes()
        return self.flat(t, T._ids_types[32], self.cfg.batch, "lengths")


def ea_recurrence(cfg, g, x, h0, lengths, y, states, h_last, workspace, stream=None):
    c, xt, gt = _Sequences(cfg), _kind(cfg.x_type, "x_type"), _kind(cfg.g_type, "g_type")
    return _check(lib.ea_recurrence(
        C.byref(cfg), c.steps(g, gt, cfg.g_stride, "g"), c.steps(x, xt, cfg.x_stride, "x"), c.ends(h0, "h0"),
        c.lengths(lengths), c.steps(y, xt, cfg.y_stride, "y"), c.states(states), c.ends(h_last, "h_last"),
        c.workspace(workspace, lib.ea_recurrence_workspace_bytes(C.byref(cfg))), c.queue(stream)))


def ea_recurrence_grad(cfg, g, x, states, lengths, dy, dh_last, dg, dx, dh0, workspace, stream=None):
    c, xt, gt = _Sequences(cfg), _kind(cfg.x_type, "x_type"), _kind(cfg.g_type, "g_type")
    return _check(lib.ea_recurrence_grad(
        C.byref(cfg), c.steps(g, gt, cfg.g_stride, "g"), c.steps(x, xt, cfg.x_stride, "x"), c.states(states),
        c.lengths(lengths), c.steps(dy, xt, cfg.y_stride, "dy"), c.ends(dh_last, "dh_last"),
        c.steps(dg, gt, cfg.g_stride, "dg"), c.steps(dx, xt, cfg.x_stride, "dx"), c.ends(dh0, "dh0"),
        c.workspace(workspace, lib.ea_recurrence_workspace_bytes(C.byref(cfg))), c.queue(stream)))


def ea_token_loss_workspace_bytes(cfg) -> int:
    return _check(lib.ea_token_loss_workspace_bytes(C.byref(cfg)))


def ea_token_loss(cfg, logits, targets, loss, total, count, dlogits, workspace, stream=None):
    c, n, kind = _Call(), cfg.rows, _kind(cfg.type, "type")
    T._dtypes()
    if cfg.index_bits not in T._ids_types:
        raise ValueError(f"index_bits must be 32 or 64 (got {cfg.index_bits})")
    return _check(lib.ea_token_loss(
        C.byref(cfg), c.rows(logits, kind, n, cfg.vocab, cfg.logits_stride, "logits"),
        c.flat(targets, T._ids_types[cfg.index_bits], n, "targets"), c.floats(loss, n, "loss"),
        c.floats(total, 1, "total"), c.flat(count, T._ids_types[32], 1, "count"),
        c.rows(dlogits, kind, n, cfg.vocab, cfg.dlogits_stride, "dlogits"),
        c.workspace(workspace, lib.ea_token_loss_workspace_bytes(C.byref(cfg))), c.queue(stream)))
