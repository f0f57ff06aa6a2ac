"""Training of the gated FFN: forward and backward pass, the norm of the gradients and the AdamW step, as functions over torch
tensors (the "training" section of sparse_ffn.h).  Every step runs in the library's kernels; torch owns the memory."""
from __future__ import annotations

import ctypes
import math
import os

import torch

from .binding import ACT_UP, _check, load_library

ACT_TRAIN = dict(ACT_UP, none=3)  # activations of either branch in training
GROUP = 256                       # entries that share the scales of their 8-bit moments
_DTYPE = {torch.float32: 0, torch.bfloat16: 1}
_vp, _i, _i64, _f64, _sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double, ctypes.c_size_t


class _TrainCall(ctypes.Structure):
    _fields_ = [("T", _i), ("D", _i), ("H", _i), ("dtype", _i), ("act", _i), ("act_up", _i), ("x", _vp), ("ld_x", _i64),
                ("W_g", _vp), ("W_up", _vp), ("W_down", _vp), ("b_g", _vp), ("z", _vp), ("u", _vp), ("ld_hidden", _i64),
                ("workspace", _vp), ("workspace_bytes", _sz), ("status", _vp)]


class _TrainGrads(ctypes.Structure):
    _fields_ = [("dx", _vp), ("ld_dx", _i64), ("dW_g", _vp), ("dW_up", _vp), ("dW_down", _vp), ("db_g", _vp)]


class _Tensor(ctypes.Structure):
    _fields_ = [("data", _vp), ("n", _i64), ("dtype", _i)]


class _AdamWTensor(ctypes.Structure):
    _fields_ = [("p", _vp), ("g", _vp), ("master", _vp), ("m", _vp), ("v", _vp), ("m_scale", _vp), ("v_scale", _vp), ("n", _i64),
                ("p_dtype", _i), ("g_dtype", _i), ("state_bits", _i), ("lr", _f64), ("weight_decay", _f64)]


class _AdamWConfig(ctypes.Structure):
    _fields_ = [("beta1", _f64), ("beta2", _f64), ("eps", _f64), ("step", _i64), ("grad_norm", _vp), ("max_norm", _f64)]


_ready = None


def _lib():
    global _ready
    if _ready is None:
        lib = load_library()
        P = ctypes.POINTER
        lib.sffn_train_workspace_bytes.argtypes = [ctypes.c_int] * 5 + [P(_sz)]
        lib.gated_ffn_forward.argtypes = [P(_TrainCall), _vp, _i64, _vp]
        lib.gated_ffn_backward.argtypes = [P(_TrainCall), _vp, _i64, P(_TrainGrads), _vp]
        lib.sffn_grad_norm.argtypes = [P(_Tensor), ctypes.c_int, _vp, _vp, _sz, _vp]
        lib.sffn_adamw_step.argtypes = [P(_AdamWTensor), ctypes.c_int, P(_AdamWConfig), _vp]
        lib.sffn_adamw_state_values.argtypes = [P(_AdamWTensor), ctypes.c_int, P(_vp), P(_vp), _vp]
        _ready = lib
    return _ready


_kept: dict = {}


def _keep(device, stream, what, nbytes):
    """A zeroed buffer of a device (of one stream, where calls that overlap may not share it) that contents outlive a call in: the
    status word, the counter of a norm."""
    key = (device.index, stream, what)
    t = _kept.get(key)
    if t is None:
        t = torch.zeros(nbytes, dtype=torch.uint8, device=device)
        if not torch.cuda.is_current_stream_capturing():  # one made while capturing is zeroed by every replay, and that graph's
            _kept[key] = t
    return t


class _On:
    """The stream a call goes to, made current for what the call allocates."""

    __slots__ = ("device", "handle", "_ctx")

    def __init__(self, device, stream):
        if device.type != "cuda":
            raise TypeError("tensors must be on a CUDA device")
        self.device = device
        self._ctx = None
        if stream is not None:
            self._ctx = torch.cuda.stream(stream)
        elif device.index != torch.cuda.current_device():
            self._ctx = torch.cuda.device(device)

    def __enter__(self):
        if self._ctx is not None:
            self._ctx.__enter__()
        self.handle = torch.cuda.current_stream(self.device).cuda_stream
        return self

    def __exit__(self, *exc):
        if self._ctx is not None:
            self._ctx.__exit__(*exc)


def _rows(name, t, shape, dtype, device):
    """A matrix of rows at one stride (in elements), consecutive entries in a row."""
    if t.shape != shape or t.dtype != dtype or t.device != device:
        raise TypeError(f"{name}: {list(shape)} {dtype} on {device} expected, got {list(t.shape)} {t.dtype} on {t.device}")
    if t.shape[1] > 1 and t.stride(1) != 1:
        raise TypeError(f"{name}: entries of a row must be consecutive")
    ld = t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1)
    return ld if t.shape[0] > 1 else -(-ld // 8) * 8


def _whole(name, t, shape, dtype, device):
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise TypeError(f"{name}: contiguous {list(shape)} {dtype} on {device} expected, got {list(t.shape)} {t.dtype} on {t.device}")
    return t.data_ptr()


def _hidden(T, H, dtype, device):
    """[T, H] with rows a multiple of 16 bytes apart."""
    return torch.empty((T, -(-H // 8) * 8), dtype=dtype, device=device)[:, :H]


def _act(name):
    return 3 if name is None else ACT_TRAIN[name]


def _call(x, W_g, b_g, W_up, W_down, act, act_up, backward, on):
    if x.dim() != 2 or W_g.dim() != 2:
        raise TypeError("x is [T, D], weights are [H, D]")
    T, D = x.shape
    H, dtype, dev = W_g.shape[0], W_g.dtype, on.device
    if dtype not in _DTYPE:
        raise TypeError("dtype must be torch.float32 or torch.bfloat16")
    c = _TrainCall(T, D, H, _DTYPE[dtype], _act(act), _act(act_up))
    c.ld_x = _rows("x", x, (T, D), dtype, dev)
    c.x = x.data_ptr()
    c.W_g, c.W_up, c.W_down = (_whole(n, w, (H, D), dtype, dev) for n, w in (("W_g", W_g), ("W_up", W_up), ("W_down", W_down)))
    if b_g is not None:
        c.b_g = _whole("b_g", b_g, (H,), torch.float32, dev)
    need = _sz(0)
    _check("sffn_train_workspace_bytes", _lib().sffn_train_workspace_bytes(T, D, H, c.dtype, int(backward), ctypes.byref(need)))
    ws = torch.empty(need.value, dtype=torch.uint8, device=dev)  # torch's blocks start on 512 bytes
    c.workspace, c.workspace_bytes = ws.data_ptr(), need.value
    status = _keep(dev, None, "status", 256)
    c.status = status.data_ptr()
    return c, (ws, status)


def training_status(device="cuda:0") -> int:
    """0, or the status that a training call on the device left because a bounded wait inside a kernel ran out (synchronises)."""
    device = torch.device(device)
    index = torch.cuda.current_device() if device.index is None else device.index
    torch.cuda.synchronize(index)
    return max([int(t[:4].view(torch.int32).item()) for (d, _, what), t in _kept.items() if d == index and what == "status"], default=0)


def _checked(name, on):
    if os.environ.get("SFFN_SYNC_CHECK") == "1" and not torch.cuda.is_current_stream_capturing():
        status = training_status(on.device)
        if status:
            raise RuntimeError(f"{name}: device status {status}")


def gated_ffn_forward(x, W_g, b_g, W_up, W_down, act="relu", act_up=None, *, save=True, y=None, z=None, u=None, stream=None):
    """y = (A(x W_g^T + b_g) * A_3(x W_up^T)) W_down over the rows of x [T, D], weights [H, D] (W_down transposed).

    Returns (y, z, u): the pre-activations z, u [T, H] are what :func:`gated_ffn_backward` needs; ``save=False`` leaves them out
    (None).  Types: x, weights, y, z, u all fp32 or all bf16, b_g fp32 or None.  ``act`` / ``act_up``: relu, sqrelu, rsplus, silu,
    none (``act_up=None``: none).  Rows of x, y, z, u may be strided (a multiple of 16 bytes)."""
    with _On(x.device, stream) as on:
        c, ws = _call(x, W_g, b_g, W_up, W_down, act, act_up, False, on)
        dtype, dev = W_g.dtype, on.device
        if y is None:
            y = torch.empty((c.T, c.D), dtype=dtype, device=dev)
        ld_y = _rows("y", y, (c.T, c.D), dtype, dev)
        if save:
            z = _hidden(c.T, c.H, dtype, dev) if z is None else z
            u = _hidden(c.T, c.H, dtype, dev) if u is None else u
            c.ld_hidden = _rows("z", z, (c.T, c.H), dtype, dev)
            if _rows("u", u, (c.T, c.H), dtype, dev) != c.ld_hidden:
                raise TypeError("z and u must have the same row stride")
            c.z, c.u = z.data_ptr(), u.data_ptr()
        else:
            z = u = None
        _check("gated_ffn_forward", _lib().gated_ffn_forward(ctypes.byref(c), y.data_ptr(), ld_y, on.handle))
        _checked("gated_ffn_forward", on)
    return y, z, u


GRADS = ("dx", "dW_g", "dW_up", "dW_down", "db_g")


def gated_ffn_backward(dy, x, z, u, W_g, W_up, W_down, act="relu", act_up=None, *, need=GRADS, out=None, stream=None):
    """Gradients of :func:`gated_ffn_forward` from dy [T, D] and what the forward pass saved: a dict of those named in ``need``
    (dx [T, D], dW_g, dW_up, dW_down [H, D] in the weights' type, db_g [H] fp32).  ``out``: a dict of tensors to write to."""
    out = dict(out or {})
    with _On(x.device, stream) as on:
        c, ws = _call(x, W_g, None, W_up, W_down, act, act_up, True, on)
        dtype, dev = W_g.dtype, on.device
        ld_dy = _rows("dy", dy, (c.T, c.D), dtype, dev)
        c.ld_hidden = _rows("z", z, (c.T, c.H), dtype, dev)
        if _rows("u", u, (c.T, c.H), dtype, dev) != c.ld_hidden:
            raise TypeError("z and u must have the same row stride")
        c.z, c.u = z.data_ptr(), u.data_ptr()
        g, got = _TrainGrads(), {}
        for name in GRADS:
            if name not in need:
                continue
            shape = (c.T, c.D) if name == "dx" else (c.H,) if name == "db_g" else (c.H, c.D)
            t = out.get(name)
            if t is None:
                t = torch.empty(shape, dtype=torch.float32 if name == "db_g" else dtype, device=dev)
            if name == "dx":
                g.ld_dx = _rows(name, t, shape, dtype, dev)
                g.dx = t.data_ptr()
            else:
                setattr(g, name, _whole(name, t, shape, torch.float32 if name == "db_g" else dtype, dev))
            got[name] = t
        unknown = set(need) - set(GRADS)
        if unknown:
            raise ValueError(f"no such gradient: {sorted(unknown)}")
        _check("gated_ffn_backward", _lib().gated_ffn_backward(ctypes.byref(c), dy.data_ptr(), ld_dy, ctypes.byref(g), on.handle))
        _checked("gated_ffn_backward", on)
    return got


class GatedFFNFunction(torch.autograd.Function):
    """The pair as a node of torch's graph: ``GatedFFNFunction.apply(x, W_g, b_g, W_up, W_down, act, act_up)``, x [..., D]."""

    @staticmethod
    def forward(ctx, x, W_g, b_g, W_up, W_down, act="relu", act_up=None):
        rows = x.reshape(-1, x.shape[-1])
        save = any(ctx.needs_input_grad)
        y, z, u = gated_ffn_forward(rows, W_g, b_g, W_up, W_down, act, act_up, save=save)
        if save:
            ctx.save_for_backward(rows, z, u, W_g, W_up, W_down)
            ctx.acts, ctx.shape = (act, act_up), x.shape
        return y.view(x.shape)

    @staticmethod
    def backward(ctx, dy):
        rows, z, u, W_g, W_up, W_down = ctx.saved_tensors
        names = ("dx", "dW_g", "db_g", "dW_up", "dW_down")
        need = [n for n, wanted in zip(names, ctx.needs_input_grad) if wanted]
        got = gated_ffn_backward(dy.reshape(rows.shape).contiguous(), rows, z, u, W_g, W_up, W_down, *ctx.acts, need=need)
        if "dx" in got:
            got["dx"] = got["dx"].view(ctx.shape)
        return (*[got.get(n) for n in names], None, None)


def _same_device(tensors):
    devices = {t.device for t in tensors}
    if len(devices) != 1:
        raise TypeError("tensors must be on one device")
    return devices.pop()


def grad_norm(tensors, norm=None, *, stream=None):
    """The 2-norm over all entries of a list of fp32 / bf16 tensors, as a 0-dimensional fp32 tensor on their device (nothing waits
    for it: hand it to :func:`adamw_step`)."""
    tensors = list(tensors)
    if not tensors:
        raise ValueError("no tensors")
    with _On(_same_device(tensors), stream) as on:
        arr = (_Tensor * len(tensors))()
        for a, t in zip(arr, tensors):
            if t.dtype not in _DTYPE or not t.is_contiguous():
                raise TypeError("gradients must be contiguous fp32 or bf16 tensors")
            a.data, a.n, a.dtype = t.data_ptr(), t.numel(), _DTYPE[t.dtype]
        if norm is None:
            norm = torch.empty((), dtype=torch.float32, device=on.device)
        out = _whole("norm", norm, torch.Size(()), torch.float32, on.device)
        ws = _keep(on.device, on.handle, "norm", 16384)
        _check("sffn_grad_norm", _lib().sffn_grad_norm(arr, len(tensors), out, ws.data_ptr(), 16384, on.handle))
    return norm


def adamw_state(p, bits=32):
    """Moments of a parameter before its first step: dict(m, v) in fp32, or with ``bits=8`` codes and their scales."""
    if bits == 32:
        return dict(m=torch.zeros_like(p, dtype=torch.float32), v=torch.zeros_like(p, dtype=torch.float32))
    if bits != 8:
        raise ValueError("moments are held in 32 or 8 bits")
    groups = -(-p.numel() // GROUP)
    return dict(m=torch.zeros_like(p, dtype=torch.int8), v=torch.zeros_like(p, dtype=torch.uint8),
                m_scale=torch.zeros(groups, device=p.device), v_scale=torch.zeros(groups, device=p.device))


def _put_state(a, state, shape, device):
    n = math.prod(shape)
    a.n = n
    if "m_scale" in state:
        a.state_bits = 8
        a.m = _whole("m", state["m"], shape, torch.int8, device)
        a.v = _whole("v", state["v"], shape, torch.uint8, device)
        groups = torch.Size((-(-n // GROUP),))
        a.m_scale = _whole("m_scale", state["m_scale"], groups, torch.float32, device)
        a.v_scale = _whole("v_scale", state["v_scale"], groups, torch.float32, device)
    else:
        a.state_bits = 32
        a.m = _whole("m", state["m"], shape, torch.float32, device)
        a.v = _whole("v", state["v"], shape, torch.float32, device)


def _each(value, n, name):
    if isinstance(value, (list, tuple)):
        if len(value) != n:
            raise ValueError(f"{name}: one value, or one for each tensor")
        return value
    return (value,) * n


def adamw_step(params, grads, states, step, *, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, masters=None, grad_norm=None,
               max_norm=None, stream=None):
    """One AdamW step over a list of tensors, in place (sffn_adamw_step): params fp32 or bf16, grads fp32 or bf16, states as
    :func:`adamw_state` makes them (updated), ``step`` = 1, 2, ...

    ``lr`` and ``weight_decay``: one number, or one for each tensor.  ``masters``: for bf16 parameters, fp32 copies that take the
    step (a list with None where there is none).  ``grad_norm``: the device scalar of :func:`grad_norm`; gradients are scaled by
    min(1, max_norm / (grad_norm + 1e-6)), and a norm that is not finite leaves everything as it was."""
    params, grads, states = list(params), list(grads), list(states)
    n = len(params)
    masters = [None] * n if masters is None else list(masters)
    if not (len(grads) == len(states) == len(masters) == n):
        raise ValueError("params, grads, states and masters must be lists of one length")
    if max_norm is not None and grad_norm is None:
        raise ValueError("max_norm needs grad_norm")
    if n == 0:
        return
    with _On(_same_device(params), stream) as on:
        arr = (_AdamWTensor * n)()
        for a, p, g, state, w, rate, decay in zip(arr, params, grads, states, masters, _each(lr, n, "lr"), _each(weight_decay, n, "weight_decay")):
            if p.dtype not in _DTYPE or g.dtype not in _DTYPE:
                raise TypeError("parameters and gradients must be fp32 or bf16")
            a.p = _whole("parameter", p, p.shape, p.dtype, on.device)
            a.g = _whole("gradient", g, p.shape, g.dtype, on.device)
            if w is not None:
                a.master = _whole("master", w, p.shape, torch.float32, on.device)
            _put_state(a, state, p.shape, on.device)
            a.p_dtype, a.g_dtype, a.lr, a.weight_decay = _DTYPE[p.dtype], _DTYPE[g.dtype], rate, decay
        c = _AdamWConfig(betas[0], betas[1], eps, step)
        if grad_norm is not None:
            c.grad_norm = _whole("grad_norm", grad_norm, torch.Size(()), torch.float32, on.device)
            c.max_norm = math.inf if max_norm is None else max_norm
        _check("sffn_adamw_step", _lib().sffn_adamw_step(arr, n, ctypes.byref(c), on.handle))


def adamw_state_values(states, out=None, *, stream=None):
    """What 8-bit moments stand for: a list of dict(m, v) in fp32 for a list of states (``out``: such a list to write to)."""
    states = list(states)
    n = len(states)
    if n == 0:
        return []
    with _On(_same_device([s["m"] for s in states]), stream) as on:
        arr, pm, pv = (_AdamWTensor * n)(), (_vp * n)(), (_vp * n)()
        if out is None:
            out = [{k: torch.empty(s["m"].shape, dtype=torch.float32, device=on.device) for k in ("m", "v")} for s in states]
        if len(out) != n:
            raise ValueError("out: one dict for each state")
        for i, (s, o) in enumerate(zip(states, out)):
            if "m_scale" not in s:
                raise TypeError("these moments are held in 32 bits")
            _put_state(arr[i], s, s["m"].shape, on.device)
            pm[i] = _whole("m", o["m"], s["m"].shape, torch.float32, on.device)
            pv[i] = _whole("v", o["v"], s["m"].shape, torch.float32, on.device)
        _check("sffn_adamw_state_values", _lib().sffn_adamw_state_values(arr, n, pm, pv, on.handle))
    return out
