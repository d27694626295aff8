"""ctypes binding of the operators beside the round (include/ea_train.h):
AdamW over many tensors, the global gradient norm, the embedding lookup and
its gradient.  Argument marshalling only, in the manner of ``_binding``: every
function has the name of the C entry point it calls, tensors are device
tensors of the documented types, streams are torch streams, raw hipStream_t
integers, or None for torch's current stream.
"""
import ctypes as C
from array import array

from . import _binding as B
from ._binding import _check, _ptr, _ptr_u32, _stream, lib

EA_F32, EA_BF16, EA_F16 = 0, 1, 2
EA_ROUND_NEAREST, EA_ROUND_STOCHASTIC = 0, 1
EA_STATE_BLOCK = 256


class Tensor(C.Structure):
    """ea_tensor_t"""
    _fields_ = [("g", C.c_void_p), ("p", C.c_void_p), ("m", C.c_void_p), ("v", C.c_void_p),
                ("m_scale", C.c_void_p), ("v_scale", C.c_void_p), ("master", C.c_void_p), ("n", C.c_int64),
                ("weight_decay", C.c_float), ("lr_scale", C.c_float)]


class AdamW(C.Structure):
    """ea_adamw_t"""
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("param_type", C.c_int32), ("grad_type", C.c_int32), ("state_bits", C.c_int32),
                ("rounding", C.c_int32), ("seed", C.c_uint64)]


class Embed(C.Structure):
    """ea_embed_t"""
    _fields_ = [("tokens", C.c_int64), ("vocab", C.c_int64), ("dim", C.c_int64), ("table_stride", C.c_int64),
                ("x_stride", C.c_int64), ("padding", C.c_int64), ("scale", C.c_float), ("table_type", C.c_int32),
                ("x_type", C.c_int32), ("index_bits", C.c_int32)]


assert C.sizeof(Tensor) == 72 and C.sizeof(AdamW) == 40 and C.sizeof(Embed) == 64

_P, _I32, _I64 = C.c_void_p, C.c_int32, C.c_int64
for _name, _res, _args in (
        ("ea_adamw_step", C.c_int, [C.POINTER(AdamW), _I64, _I32, _P, _P, _P]),
        ("ea_adamw_step_scheduled", C.c_int, [C.POINTER(AdamW), C.POINTER(B.Schedule), _P, _I32, _P, _P, _P]),
        ("ea_grad_norm_workspace_bytes", _I64, [_I32, _P]),
        ("ea_grad_norm", C.c_int, [_I32, _I32, _P, C.c_float, C.c_float, _P, _P, _P, _P]),
        ("ea_embed_lookup", C.c_int, [C.POINTER(Embed), _P, _P, _P, _P]),
        ("ea_embed_workspace_bytes", _I64, [C.POINTER(Embed)]),
        ("ea_embed_grad", C.c_int, [C.POINTER(Embed), _P, _P, _P, _I32, _P, _P])):
    getattr(lib, _name).restype, getattr(lib, _name).argtypes = _res, _args


# torch's dtypes by EA_F32, EA_BF16, EA_F16, its integer dtypes by bits, and the current device's number;
# looked up on first use.  A small call takes the GPU 2 to 3 us and a launch the host 3.5, so what a call checks
# is kept short (from Python, AdamW on four tensors 6.2 -> 5.9 us a call, a lookup 7.0 -> 6.0).
_types = _ids_types = _current = None


def _dtypes():
    global _types, _ids_types, _current
    if _types is None:
        import torch
        if B._torch is None:
            B._load_torch()
        _ids_types = {32: torch.int32, 64: torch.int64}
        _current = getattr(torch._C, "_cuda_getDevice", None) or B._device
        _types = (torch.float32, torch.bfloat16, torch.float16)
    return _types


def ea_type(dtype) -> int:
    """EA_F32, EA_BF16 or EA_F16 for a torch dtype."""
    if dtype not in _dtypes():
        raise ValueError(f"libea takes float32, bfloat16 or float16 here, got {dtype}")
    return _types.index(dtype)


def _dense(t) -> bool:
    """Whether the tensor fills its memory without gaps or overlaps, in any order."""
    if t.is_contiguous():
        return True
    expect = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if stride != expect:
            return False
        expect *= size
    return True


def _same_order(t, e) -> bool:
    """Whether two tensors of one shape go through their elements in the same order of memory."""
    return t.stride() == e.stride() or all(a == b for a, b, n in zip(t.stride(), e.stride(), t.shape) if n != 1)


def _is_tensor(name, i, t):
    if not hasattr(t, "data_ptr"):
        raise ValueError(f"{name}[{i}]: expected a tensor, got {type(t).__name__}")


def _each(name, x, n):
    """n numbers from one for all, or from a sequence of n."""
    if isinstance(x, (int, float)) or getattr(x, "ndim", 1) == 0:
        return [x] * n
    if len(x) != n:
        raise ValueError(f"{len(x)} values of {name}, and {n} tensors")
    return x


class TensorList:
    """The tensors of an AdamW step or a gradient norm: an ea_tensor_t array and references to what it points
    to.  A program makes it once and passes it every step; ``set_grads`` replaces the gradients.  It stands for
    the memory that the tensors had when it was made: one whose storage is replaced (``t.data = ...``) needs a new list.

    g, p, m, v, m_scale, v_scale, master: lists of device tensors, one per parameter (all but g may be None;
    entries of master too).  g, p and master of a parameter share its shape and strides and are dense; m and v
    hold its number of elements in the same memory order, as float32, or as 8-bit codes (float8_e4m3fn or
    uint8) with scales.  weight_decay, lr_scale: one number, or one per parameter.
    """

    def __init__(self, g, p=None, m=None, v=None, m_scale=None, v_scale=None, master=None, weight_decay=0.0,
                 lr_scale=1.0):
        n = len(g)
        self.count = n
        self.array = (Tensor * max(n, 1))()
        self.address = C.addressof(self.array)
        self._words = memoryview(self.array).cast("B").cast("Q")   # a field of all tensors: every 9th word
        self.param_type = self.grad_type = self.state_bits = self._n = None
        self._p = None if p is None else tuple(p)
        for name, ts in (("p", p), ("m", m), ("v", v), ("m_scale", m_scale), ("v_scale", v_scale),
                         ("master", master)):
            if ts is not None and len(ts) != n:
                raise ValueError(f"{len(ts)} tensors in {name}, and {n} in g")
        for i, t in enumerate(p or ()):
            _is_tensor("p", i, t)
        self.set_grads(g)
        if p is not None:
            self.param_type, at = self._checked("p", p, g)
            self._column("p", at)
            if master is not None:
                self._column("master", self._checked("master", master, p, _dtypes()[EA_F32], optional=True)[1])
        if (m is None) != (v is None):
            raise ValueError("m and v come together")
        if m is not None:
            self.state_bits = self._set_states(m, v, m_scale, v_scale)
        for e, wd, ls in zip(self.array, _each("weight_decay", weight_decay, n), _each("lr_scale", lr_scale, n)):
            e.weight_decay, e.lr_scale = wd, ls
        self.kinds = (self.param_type, self.grad_type, self.state_bits)
        self.norm_bytes = _check(lib.ea_grad_norm_workspace_bytes(n, self.address))
        # the memory stays, whatever becomes of the caller's lists and tensors (the gradients': set_grads)
        self._held = [t.untyped_storage() for ts in (p, m, v, m_scale, v_scale, master) if ts is not None
                      for t in ts if t is not None]
        if p is not None:
            at = [t.data_ptr() for t in p if t.numel()]
            if len(set(at)) != len(at):
                raise ValueError("a parameter is in the list twice")

    def _column(self, name, values):
        if values:
            self._words[getattr(Tensor, name).offset // 8::C.sizeof(Tensor) // 8] = array("Q", values)

    def _checked(self, name, ts, like, dtype=None, optional=False):
        """`name`'s tensors checked against those of `like`: (their type, their addresses)."""
        if ts and all(hasattr(t, "data_ptr") for t in ts) and len({t.dtype for t in ts}) == 1 and \
                (dtype is None or ts[0].dtype is dtype) and {t.get_device() for t in ts} == {like[0].get_device()} and \
                ts[0].is_cuda and all(t.is_contiguous() for t in ts) and \
                (ts is like or all(t.shape == e.shape and e.is_contiguous() for t, e in zip(ts, like))):
            return ea_type(ts[0].dtype), [t.data_ptr() for t in ts]
        # other strides, a part of the entries, or something to refuse: one by one
        kind, at = None, []
        for i, t in enumerate(ts):
            if t is None and optional:
                at.append(0)
                continue
            _is_tensor(name, i, t)
            if dtype is not None and t.dtype is not dtype:
                raise ValueError(f"{name}[{i}]: expected {dtype}, got {t.dtype}")
            if kind is None:
                kind = t.dtype
            elif t.dtype is not kind:
                raise ValueError(f"{name}[{i}]: all of {name} share one type, got {t.dtype} after {kind}")
            if not t.is_cuda:
                raise ValueError("libea needs device tensors")
            e = like[i]
            if e is not t:
                if t.get_device() != e.get_device():
                    raise ValueError(f"{name}[{i}] is on {t.device}, and others on {e.device}")
                if t.shape != e.shape or (t.numel() > 1 and not _same_order(t, e)):
                    raise ValueError(f"{name}[{i}]: shape {tuple(t.shape)}, strides {t.stride()} are not the "
                                     f"parameter's {tuple(e.shape)}, {e.stride()}")
            if not t.is_contiguous() and not _dense(t):
                raise ValueError(f"{name}[{i}]: strides {t.stride()} leave gaps in shape {tuple(t.shape)}")
            at.append(t.data_ptr())
        return None if kind is None else ea_type(kind), at

    def _set_states(self, m, v, m_scale, v_scale):
        import torch
        codes = (torch.float8_e4m3fn, torch.uint8)
        bits = 8 if self.count and getattr(m[0], "dtype", None) in codes else 32
        if bits == 8 and (m_scale is None or v_scale is None):
            raise ValueError("8-bit states come with m_scale and v_scale")
        for name, ts in (("m", m), ("v", v), ("m_scale", m_scale), ("v_scale", v_scale)):
            if ts is None or (bits == 32 and name.endswith("scale")):
                continue
            want = codes if bits == 8 and name in "mv" else (torch.float32,)
            per = 1 if name in "mv" else EA_STATE_BLOCK
            for i, t in enumerate(ts):
                most = (self._n[i] + per - 1) // per
                _is_tensor(name, i, t)
                if not t.is_cuda:
                    raise ValueError("libea needs device tensors")
                if t.dtype not in want or t.numel() != most or t.device != self._g[i].device or \
                        not (t.is_contiguous() or _dense(t)):
                    raise ValueError(f"{name}[{i}]: expected {most} dense elements of {want[0]} on the gradient's "
                                     f"device, got {t.numel()} of {t.dtype} on {t.device}")
            self._column(name, [t.data_ptr() for t in ts])
        return bits

    def set_grads(self, g):
        """Points the list at other gradients of the same shapes."""
        if len(g) != self.count:
            raise ValueError(f"{len(g)} gradients for {self.count} tensors")
        kind, at = self._checked("g", g, g if self._p is None else self._p)
        if self.grad_type is not None and kind != self.grad_type:
            raise ValueError("the gradients' type changed")
        sizes, devices = [t.numel() for t in g], {t.get_device() for t in g}
        if self._n is not None and sizes != self._n:
            raise ValueError("the gradients' sizes changed")
        if len(devices) > 1:
            raise ValueError("the tensors are not all on one device")
        self._n = sizes
        self._column("n", sizes)
        self._column("g", at)
        self.grad_type, self.device = kind, devices.pop() if devices else None
        self._g, self._g_held = tuple(g), [t.untyped_storage() for t in g]


def _queue(stream, device):
    """The raw stream of a call on tensors of `device`, which has to be the current one."""
    if _types is None:
        _dtypes()
    here = _current() if device is not None else B._device()
    if device != here and device is not None:
        raise ValueError(f"the tensors are on device {device}, and the current device is {here}")
    return B._raw_stream(here) if stream is None and B._raw_stream else _stream(stream)


def _check_list(cfg, tensors):
    if tensors.param_type is None or tensors.state_bits is None:
        raise ValueError("a step needs p, m and v")
    raise ValueError(f"the tensors' types (param {tensors.param_type}, grad {tensors.grad_type}, states "
                     f"{tensors.state_bits} bits) are not the configuration's ({cfg.param_type}, "
                     f"{cfg.grad_type}, {cfg.state_bits} bits)")


def _one(t, device, name):
    """Pointer of a scalar (float32, but for t_dev) on the list's device."""
    if t is None or isinstance(t, int):
        return t
    at = _ptr_u32(t) if name == "t_dev" else _ptr(t, B._F32)
    if t.numel() < 1:
        raise ValueError(f"{name}: expected one element, got none")
    if device is not None and t.get_device() != device:
        raise ValueError(f"{name} is on {t.device}, and the list's tensors on device {device}")
    return at


def ea_adamw_step(cfg, t, tensors, gscale=None, stream=None):
    if tensors.kinds != (cfg.param_type, cfg.grad_type, cfg.state_bits) and tensors.count:
        _check_list(cfg, tensors)
    queue = _queue(stream, tensors.device)
    return _check(lib.ea_adamw_step(C.byref(cfg), t, tensors.count, tensors.address,
                                    None if gscale is None else _one(gscale, tensors.device, "gscale"), queue))


def ea_adamw_step_scheduled(cfg, sched, t_dev, tensors, gscale=None, stream=None):
    if tensors.kinds != (cfg.param_type, cfg.grad_type, cfg.state_bits) and tensors.count:
        _check_list(cfg, tensors)
    queue = _queue(stream, tensors.device)
    return _check(lib.ea_adamw_step_scheduled(C.byref(cfg), C.byref(sched), _one(t_dev, tensors.device, "t_dev"),
                                              tensors.count, tensors.address, _one(gscale, tensors.device, "gscale"),
                                              queue))


def ea_grad_norm_workspace_bytes(tensors) -> int:
    return _check(lib.ea_grad_norm_workspace_bytes(tensors.count, tensors.address))


def ea_grad_norm(tensors, scale, max_norm, norm, gscale, workspace, stream=None):
    queue = _queue(stream, tensors.device)
    d = tensors.device
    _room(workspace, tensors.norm_bytes)
    if d is not None and hasattr(workspace, "get_device") and workspace.is_cuda and workspace.get_device() != d:
        raise ValueError(f"the workspace is on {workspace.device}, and the list's tensors on device {d}")
    return _check(lib.ea_grad_norm(tensors.grad_type or EA_F32, tensors.count, tensors.address, scale, max_norm,
                                   _one(norm, d, "norm"), _one(gscale, d, "gscale"), _ptr(workspace), queue))


def _room(workspace, need):
    if need < 0:
        raise B.EAError(need, B.ea_last_error())
    if need > 0 and hasattr(workspace, "numel") and workspace.numel() * workspace.element_size() < need:
        raise ValueError(f"the workspace holds {workspace.numel() * workspace.element_size()} bytes, {need} are needed")


def _rows(t, kind, rows, dim, stride, name):
    """Pointer of a [rows, dim] tensor (leading dimensions may be split) with `stride` elements between rows."""
    if t is None or isinstance(t, int):
        return t
    if not t.is_cuda:
        raise ValueError("libea needs device tensors")
    if ea_type(t.dtype) != kind:
        raise ValueError(f"{name}: {t.dtype} is not the configuration's type {kind}")
    if t.dim() < 1 or t.shape[-1] != dim or t.numel() != rows * dim:
        raise ValueError(f"{name}: expected {rows} rows of {dim}, got shape {tuple(t.shape)}")
    if t.numel() == 0:
        return t.data_ptr()
    step = stride
    for k in range(t.dim() - 2, -1, -1):
        if t.shape[k] != 1 and t.stride(k) != step:
            raise ValueError(f"{name}: strides {t.stride()} are not those of rows {stride} elements apart")
        step *= t.shape[k]
    if dim > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row are not next to each other")
    return t.data_ptr()


def _ids(t, cfg):
    if t is None or isinstance(t, int):
        return t
    if t.is_floating_point() or t.is_complex() or t.element_size() * 8 != cfg.index_bits:
        raise ValueError(f"ids: expected {cfg.index_bits}-bit integers, got {t.dtype}")
    if t.numel() != cfg.tokens:
        raise ValueError(f"ids: expected {cfg.tokens}, got {t.numel()}")
    return _ptr(t)


def _device_of(*tensors):
    """The one device of these tensors (raw pointers and None left out)."""
    got = {t.get_device() for t in tensors if hasattr(t, "get_device") and t.is_cuda}
    if len(got) > 1:
        raise ValueError("the tensors are not all on one device")
    return got.pop() if got else None


def _fits(cfg, table, ids, x):
    """Whether three tensors are what the configuration says, the plain way; anything else is looked at in turn."""
    try:
        dim, device, types = cfg.dim, table.get_device(), _types or _dtypes()
        return device >= 0 and x.get_device() == device and ids.get_device() == device and \
            table.dtype is types[cfg.table_type] and x.dtype is types[cfg.x_type] and \
            ids.dtype is _ids_types[cfg.index_bits] and ids.is_contiguous() and ids.numel() == cfg.tokens and \
            table.shape == (cfg.vocab, dim) and table.stride() == (cfg.table_stride, 1) and \
            x.shape == (cfg.tokens, dim) and x.stride() == (cfg.x_stride, 1)
    except (AttributeError, IndexError, KeyError):
        return False


def ea_embed_lookup(cfg, table, ids, x, stream=None):
    if _fits(cfg, table, ids, x):
        return _check(lib.ea_embed_lookup(C.byref(cfg), table.data_ptr(), ids.data_ptr(), x.data_ptr(),
                                          _queue(stream, table.get_device())))
    args = (_rows(table, cfg.table_type, cfg.vocab, cfg.dim, cfg.table_stride, "table"), _ids(ids, cfg),
            _rows(x, cfg.x_type, cfg.tokens, cfg.dim, cfg.x_stride, "x"))
    return _check(lib.ea_embed_lookup(C.byref(cfg), *args, _queue(stream, _device_of(table, ids, x))))


def ea_embed_workspace_bytes(cfg) -> int:
    return _check(lib.ea_embed_workspace_bytes(C.byref(cfg)))


def ea_embed_grad(cfg, ids, dx, dtable, accumulate, workspace, stream=None):
    _room(workspace, lib.ea_embed_workspace_bytes(C.byref(cfg)))
    if _fits(cfg, dtable, ids, dx) and (not hasattr(workspace, "get_device") or
                                        workspace.get_device() == dx.get_device()):
        return _check(lib.ea_embed_grad(C.byref(cfg), ids.data_ptr(), dx.data_ptr(), dtable.data_ptr(),
                                        1 if accumulate else 0, _ptr(workspace), _queue(stream, dx.get_device())))
    args = (_ids(ids, cfg), _rows(dx, cfg.x_type, cfg.tokens, cfg.dim, cfg.x_stride, "dx"),
            _rows(dtable, cfg.table_type, cfg.vocab, cfg.dim, cfg.table_stride, "dtable"), 1 if accumulate else 0,
            _ptr(workspace))
    return _check(lib.ea_embed_grad(C.byref(cfg), *args, _queue(stream, _device_of(ids, dx, dtable, workspace))))
