"""The Muon optimiser for the matrices of a model (the "Muon" section of sparse_ffn.h): an update made orthogonal by Newton-Schulz
products, and the whole step over a list of matrices.  What is not a matrix (biases, gains) takes :func:`adamw_step`."""
from __future__ import annotations

import math

import torch

from .binding import SFFNError
from .training import _calls, _checked, _keep, _looked_at

MUON_COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _flat(coefficients, steps):
    """Three numbers for every step, from one triple or a triple a step."""
    if steps < 1:
        raise ValueError("at least one step")
    triples = [tuple(c) for c in coefficients] if hasattr(coefficients[0], "__len__") else [tuple(coefficients)] * steps
    if len(triples) != steps or any(len(t) != 3 for t in triples):
        raise ValueError("coefficients: one triple, or one for every step")
    return [float(v) for t in triples for v in t]


def _device(tensors, what):
    if not tensors:
        return None
    if not isinstance(tensors[0], torch.Tensor) or not tensors[0].is_cuda:
        raise TypeError(f"{what}: tensors on a CUDA device expected")
    return tensors[0].device


def orthogonalize(update, out=None, *, steps=5, coefficients=MUON_COEFFICIENTS, eps=1e-7, bits=None, stream=None):
    """The orthogonal matrix of an update [rows, cols] (or a list of them, for a list): X = U / (|U| + eps), then ``steps`` times
    X = a X + (b P + c P^2) X with P = X X^T on the shorter side.  fp32 or bf16; rows may be strided.

    ``coefficients``: (a, b, c), or one such triple for every step.  ``bits`` of the products' operands: 16 (one fp16 term, O within
    about 1e-3 of its norm besides its own rounding, 3e-3 where a side is below 16, 5e-3 where singular values are few or far apart), 32
    (two terms, within 2e-5, three products for one; of a matrix with a null space up to 5e-4, as fp32 products), None: 16 for bf16, 32
    for fp32.  ``out``: a tensor (a list) to write to, which may be the update itself."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return orthogonalize(update, out, steps=steps, coefficients=coefficients, eps=eps, bits=bits)
    if isinstance(update, torch.Tensor):
        return orthogonalize([update], None if out is None else [out], steps=steps, coefficients=coefficients, eps=eps, bits=bits)[0]
    updates = list(update)
    device = _device(updates, "orthogonalize")
    if device is None:
        return []
    rc, got = _calls().orthogonalize(updates, None if out is None else list(out), _flat(coefficients, steps), eps, bits or 0,
                                     _keep(device.index, None, "status", 256))
    if rc or _looked_at():
        _checked("sffn_orthogonalize", rc, device)
    return got


def muon_state(p):
    """What a matrix keeps between steps, before its first one: dict(m) in fp32."""
    return dict(m=torch.zeros_like(p, dtype=torch.float32, memory_format=torch.contiguous_format))


def _scale(rule, p):
    """A step's size by rule: "spectral" sqrt(max(1, rows / cols)), "rms" 0.2 sqrt(max(rows, cols)) (entries as large as AdamW's)."""
    if not isinstance(rule, str):
        return float(rule)
    rows, cols = p.shape
    if rule == "spectral":
        return math.sqrt(max(1.0, rows / cols)) if cols else 1.0
    if rule == "rms":
        return 0.2 * math.sqrt(max(rows, cols))
    raise ValueError(f"scale: a number, 'spectral' or 'rms', not {rule!r}")


def muon_step(params, grads, states, *, lr, momentum=0.95, nesterov=True, weight_decay=0.01, scale="spectral", steps=5, coefficients=MUON_COEFFICIENTS,
              eps=1e-7, bits=None, masters=None, grad_norm=None, max_norm=None, stream=None):
    """One Muon step over a list of matrices, in place (sffn_muon_step): m = momentum m + (1 - momentum) g, U = (1 - momentum) g + momentum m
    (``nesterov=False``: m), p = p (1 - lr weight_decay) - lr scale O, O the orthogonal matrix of U (:func:`orthogonalize`).

    params fp32 or bf16 matrices, grads fp32 or bf16, states as :func:`muon_state` makes them (updated).  ``lr``, ``weight_decay`` and
    ``scale``: one for all, or one for each; scale a number, "spectral" or "rms".  ``masters``: for bf16 parameters, fp32 copies that
    take the step (a list with None where there is none).  ``bits`` of the products: None: 32 where a parameter or its master is fp32,
    else 16, which takes a third of the time (how far off either is: :func:`orthogonalize`).  ``grad_norm``, ``max_norm``: as for :func:`adamw_step`: a
    norm that is not finite leaves everything as it was.  Calls that read the parameters may follow on the same stream."""
    if max_norm is not None and grad_norm is None:
        raise ValueError("max_norm needs grad_norm")
    if stream is not None:
        with torch.cuda.stream(stream):
            return muon_step(params, grads, states, lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, scale=scale, steps=steps,
                             coefficients=coefficients, eps=eps, bits=bits, masters=masters, grad_norm=grad_norm, max_norm=max_norm)
    params, grads, states, masters = [v if v is None or isinstance(v, (list, tuple)) else list(v) for v in (params, grads, states, masters)]
    device = _device(params, "muon_step")
    if device is None:
        if grads or states or masters:
            raise ValueError("params, grads, states and masters must be lists of one length")
        return
    for p in params:
        if not isinstance(p, torch.Tensor) or p.dim() != 2:
            raise TypeError("muon_step takes matrices: biases and gains go to adamw_step")
    rules = list(scale) if isinstance(scale, (list, tuple)) else [scale] * len(params)
    if len(rules) != len(params):
        raise ValueError("scale: one value, or one for each tensor")
    rc = _calls().muon_step(params, grads, states, masters, lr, momentum, nesterov, weight_decay, [_scale(r, p) for r, p in zip(rules, params)],
                            _flat(coefficients, steps), eps, bits or 0, grad_norm, math.inf if max_norm is None else max_norm,
                            _keep(device.index, None, "status", 256))
    if rc or _looked_at():
        _checked("sffn_muon_step", rc, device)
