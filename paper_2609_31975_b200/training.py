"""Training of the gated FFN: forward and backward pass, the norm of the gradients and the AdamW step, as functions over torch
tensors (the "training" section of sparse_ffn.h).  Every step runs in the library's kernels; torch owns the memory.  Arguments are
checked and marshalled in C++ (csrc/torch_calls.cpp).  A call that writes into a caller's tensor counts as an operation in place: a
backward pass of torch's graph that saved the tensor before raises."""
from __future__ import annotations

import ctypes
import math
import os

import torch

from .binding import _SYNC_CHECK, ACT_UP, SFFNError, _environ, _raw_stream, _variables, load_library

ACT_TRAIN = dict(ACT_UP, none=3)  # activations of either branch in training
ACT_TRAIN[None] = 3
GROUP = 256                       # entries that share the scales of their 8-bit moments
_ENTRIES = ("sffn_train_workspace_bytes", "gated_ffn_forward", "gated_ffn_backward", "sffn_grad_norm", "sffn_adamw_step",
            "sffn_adamw_state_values")

_bound = None


def _calls():
    """The compiled side of this module, bound to the library's entry points; raises if it has not been built."""
    global _bound
    if _bound is None:
        lib = load_library()
        try:
            from . import _training
        except ImportError as e:
            raise RuntimeError("_training.so is missing or does not load: build it with `python -m paper_2609_31975_b200.build`") from e
        if _training.torch_version != torch.__version__:
            raise RuntimeError(f"_training.so was built for torch {_training.torch_version}: build it with `python -m paper_2609_31975_b200.build`")
        _training.bind([ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _ENTRIES])
        _bound = _training
    return _bound


_kept: dict = {}


def _keep(index, stream, what, nbytes):
    """A zeroed buffer of a device (of one stream, where calls that overlap may not share it) whose contents outlive a call: the
    status word, the counter of a norm."""
    t = _kept.get((index, stream, what))
    if t is None:
        if index < 0:
            raise TypeError("tensors must be on a CUDA device")
        t = _kept[index, stream, what] = _calls().kept(nbytes, index)
    return t


def training_status(device="cuda:0", reset=False) -> int:
    """0, or the status that a training call on the device left because a bounded wait inside a kernel ran out (synchronises).  It
    stays until ``reset``; what such a call was to write is not to be used."""
    device = torch.device(device)
    index = torch.cuda.current_device() if device.index is None else device.index
    torch.cuda.synchronize(index)
    word = _kept.get((index, None, "status"))
    status = 0 if word is None else int(word[:4].view(torch.int32).item())
    if reset and word is not None:
        word.zero_()
        torch.cuda.synchronize(index)
    return status


def _looked_at():
    """Whether SFFN_SYNC_CHECK may be set: os.environ itself is asked only where it may (see binding.py)."""
    return _SYNC_CHECK in _variables or os.environ is not _environ


def _checked(name, rc, device):
    if rc:
        raise SFFNError(name, rc)
    if os.environ.get("SFFN_SYNC_CHECK") == "1" and not torch.cuda.is_current_stream_capturing():
        status = training_status(device)
        if status:
            raise RuntimeError(f"{name}: device status {status}")


def gated_ffn_forward(x, W_g, b_g, W_up, W_down, act="relu", act_up=None, *, save=True, y=None, z=None, u=None, stream=None):
    """y = (A(x W_g^T + b_g) * A_3(x W_up^T)) W_down over the rows of x [T, D], weights [H, D] (W_down transposed).

    Returns (y, z, u): the pre-activations z, u [T, H] are what :func:`gated_ffn_backward` needs; ``save=False`` leaves them out
    (None).  Types: x, weights, y, z, u all fp32 or all bf16, b_g fp32 or None.  ``act`` / ``act_up``: relu, sqrelu, rsplus, silu,
    none (``act_up=None``: none).  Rows of x, y, z, u may be strided (a multiple of 16 bytes).  y may be x; no other output may
    share memory with an input or another output."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return gated_ffn_forward(x, W_g, b_g, W_up, W_down, act, act_up, save=save, y=y, z=z, u=u)
    rc, y, z, u = _calls().ffn_forward(x, W_g, b_g, W_up, W_down, ACT_TRAIN[act], ACT_TRAIN[act_up], save, y, z, u,
                                       _keep(x.get_device(), None, "status", 256))
    if rc or _looked_at():
        _checked("gated_ffn_forward", rc, x.device)
    return y, z, u


GRADS = ("dx", "dW_g", "dW_up", "dW_down", "db_g")


def gated_ffn_backward(dy, x, z, u, W_g, W_up, W_down, act="relu", act_up=None, *, need=GRADS, out=None, stream=None):
    """Gradients of :func:`gated_ffn_forward` from dy [T, D] and what the forward pass saved: a dict of those named in ``need``
    (dx [T, D], dW_g, dW_up, dW_down [H, D] in the weights' type, db_g [H] fp32).  ``out``: a dict of tensors to write to (those
    not in ``need`` are left alone); dx may be dy, x, z or u, no other one may share memory with an input or another output."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return gated_ffn_backward(dy, x, z, u, W_g, W_up, W_down, act, act_up, need=need, out=out)
    if out and set(out) - set(GRADS):
        raise ValueError(f"no such gradient: {sorted(set(out) - set(GRADS))}")
    bits = 31
    if need is not GRADS:
        bits = sum(1 << GRADS.index(name) for name in set(need) if name in GRADS)
        if set(need) - set(GRADS):
            raise ValueError(f"no such gradient: {sorted(set(need) - set(GRADS))}")
    rc, *got = _calls().ffn_backward(dy, x, z, u, W_g, W_up, W_down, ACT_TRAIN[act], ACT_TRAIN[act_up], bits,
                                     [out.get(name) for name in GRADS] if out else [], _keep(x.get_device(), None, "status", 256))
    if rc or _looked_at():
        _checked("gated_ffn_backward", rc, x.device)
    return {name: t for name, t in zip(GRADS, got) if t is not None}


class GatedFFNFunction(torch.autograd.Function):
    """The pair as a node of torch's graph: ``GatedFFNFunction.apply(x, W_g, b_g, W_up, W_down, act, act_up)``, x [..., D].
    First derivatives only: a second differentiation (``create_graph=True``, then through the gradients) raises."""

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
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        rows, z, u, W_g, W_up, W_down = ctx.saved_tensors
        names = ("dx", "dW_g", "db_g", "dW_up", "dW_down")
        need = [n for n, wanted in zip(names, ctx.needs_input_grad) if wanted]
        dy = dy.reshape(rows.shape).contiguous()
        if dy.data_ptr() % 16:  # a slice of something longer
            dy = dy.clone()
        got = gated_ffn_backward(dy, rows, z, u, W_g, W_up, W_down, *ctx.acts, need=need)
        if "dx" in got:
            got["dx"] = got["dx"].view(ctx.shape)
        return (*[got.get(n) for n in names], None, None)


def grad_norm(tensors, norm=None, *, stream=None):
    """The 2-norm over all entries of a list of fp32 / bf16 tensors, as a 0-dimensional fp32 tensor on their device (nothing waits
    for it: hand it to :func:`adamw_step`)."""
    if not isinstance(tensors, (list, tuple)):
        tensors = list(tensors)
    if not tensors:
        raise ValueError("no tensors")
    if stream is not None:
        with torch.cuda.stream(stream):
            return grad_norm(tensors, norm)
    index = tensors[0].get_device()
    rc, norm = _calls().grad_norm(tensors, norm, _keep(index, _raw_stream(index) if index >= 0 else None, "norm", 16384))
    if rc:
        raise SFFNError("sffn_grad_norm", rc)
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


def adamw_step(params, grads, states, step, *, lr, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, masters=None, grad_norm=None,
               max_norm=None, stream=None):
    """One AdamW step over a list of tensors, in place (sffn_adamw_step): params fp32 or bf16, grads fp32 or bf16, states as
    :func:`adamw_state` makes them (updated), ``step`` = 1, 2, ...

    ``eps`` may be 0, with 8-bit moments 8.9e-16 at least.  ``lr`` and ``weight_decay``: one number, or one for each tensor.  ``masters``: for bf16 parameters, fp32 copies that take the
    step (a list with None where there is none).  ``grad_norm``: the device scalar of :func:`grad_norm`; gradients are scaled by
    min(1, max_norm / (grad_norm + 1e-6)), and a norm that is not finite leaves everything as it was.  Calls that read the parameters,
    :meth:`SparseFFN.sparse_ffn_forward` too, may follow on the same stream without a synchronisation."""
    if max_norm is not None and grad_norm is None:
        raise ValueError("max_norm needs grad_norm")
    if stream is not None:
        with torch.cuda.stream(stream):
            return adamw_step(params, grads, states, step, lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, masters=masters,
                              grad_norm=grad_norm, max_norm=max_norm)
    lists = [v if v is None or isinstance(v, (list, tuple)) else list(v) for v in (params, grads, states, masters)]
    rc = _calls().adamw_step(*lists, step, lr, betas[0], betas[1], eps, weight_decay, grad_norm, math.inf if max_norm is None else max_norm)
    if rc:
        raise SFFNError("sffn_adamw_step", rc)


def adamw_state_values(states, out=None, *, stream=None):
    """What 8-bit moments stand for: a list of dict(m, v) in fp32 for a list of states (``out``: such a list to write to)."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return adamw_state_values(states, out)
    states = list(states)
    if out is None:
        out = [{k: torch.empty(s["m"].shape, dtype=torch.float32, device=s["m"].device) for k in ("m", "v")} for s in states]
    rc = _calls().adamw_state_values(states, out)
    if rc:
        raise SFFNError("sffn_adamw_state_values", rc)
    return out
