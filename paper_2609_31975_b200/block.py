"""The norms before and after a block of a residual stream, with its gate, its residual scale and the sum (the "block" section of
sparse_ffn.h): forward and backward pass as functions over torch tensors, and a node of torch's graph.  A row is a token: the same
call serves a training batch and one decoded token, whose fp32 FFN output goes onto a bf16 stream."""
from __future__ import annotations

import torch

from .binding import SFFNError
from .training import _calls

BLOCK_GRADS = ("dy", "dresid", "dpost_gain", "dpre_gain", "dgate")


def block_norm_forward(y, resid, post_gain=None, pre_gain=None, gate=None, *, scale=1.0, eps=1e-6, save=True, h_dtype=None, n_dtype=None, h=None, n=None,
                       stream=None):
    """h = resid + scale * gate * N(y; post_gain) and n = N(h; pre_gain), with N(v; g) = v / sqrt(mean(v^2) + eps) * g over the rows.

    Returns (h, n, stats); stats [2, T] is what :func:`block_norm_backward` needs (``save=False``: None).  ``post_gain`` None: y is
    taken as it is; ``pre_gain`` None: there is no n (None); ``resid`` None: h is the second term; ``y`` None: h is resid itself, n its
    norm.  y, resid [T, D] (or [D], one token); each of y, resid and h, n may be fp32 or bf16: h has resid's type (without resid
    ``h_dtype``, or y's), n ``n_dtype``, or h's.  Gains [D] fp32.  ``gate``: [D] or [T, 1] fp32, or [T, D] of h's type.  Rows may be
    strided (a multiple of 16 bytes).  ``h`` and ``n``: tensors to write to; h may be resid, no other output may share memory with an
    input or another output."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return block_norm_forward(y, resid, post_gain, pre_gain, gate, scale=scale, eps=eps, save=save, h_dtype=h_dtype, n_dtype=n_dtype, h=h, n=n)
    like = y if resid is None else resid
    if like is not None and like.dim() == 1:  # one token
        one = lambda t: None if t is None else t[None]  # noqa: E731
        got_h, got_n, stats = block_norm_forward(one(y), one(resid), post_gain, pre_gain, gate, scale=scale, eps=eps, save=save, h_dtype=h_dtype,
                                                 n_dtype=n_dtype, h=one(h), n=one(n))
        return got_h[0], None if got_n is None else got_n[0], stats
    rc, got_h, got_n, stats = _calls().block_forward(y, resid, post_gain, pre_gain, gate, scale, eps, save, h_dtype, n_dtype, h, n)
    if rc:
        raise SFFNError("sffn_block_norm_forward", rc)
    return resid if y is None else got_h, got_n, stats


def block_norm_backward(dh, dn, y, h, stats, post_gain=None, pre_gain=None, gate=None, *, scale=1.0, need=BLOCK_GRADS, out=None, stream=None):
    """Gradients of :func:`block_norm_forward` from dh (h's type) and dn (n's type; either may be None), y, and the h and stats that the
    forward pass left: a dict of those named in ``need`` that the call has (dy, dresid [T, D]; dpost_gain, dpre_gain [D] fp32; dgate as
    the gate).  ``out``: a dict of tensors to write to (those not in ``need`` are left alone); dresid may be dh, no other one may share
    memory with an input or another output."""
    if stream is not None:
        with torch.cuda.stream(stream):
            return block_norm_backward(dh, dn, y, h, stats, post_gain, pre_gain, gate, scale=scale, need=need, out=out)
    bits = 31
    if need is not BLOCK_GRADS or out:
        need = tuple(need)
        for name in (*need, *(out or ())):
            if name not in BLOCK_GRADS:
                raise ValueError(f"no such gradient: {name!r}")
        bits = sum(1 << BLOCK_GRADS.index(name) for name in set(need))
    if dh is None and dn is None:
        raise ValueError("dh or dn is needed")
    if h.dim() == 1:  # one token
        one = lambda t: None if t is None else t[None]  # noqa: E731
        rows = {k: t[None] if k in ("dy", "dresid") else t for k, t in (out or {}).items()}
        got = block_norm_backward(one(dh), one(dn), one(y), h[None], stats, post_gain, pre_gain, gate, scale=scale, need=need, out=rows)
        return {k: t[0] if k in ("dy", "dresid") else t for k, t in got.items()}
    rc, *got = _calls().block_backward(dh, dn, y, h, stats, post_gain, pre_gain, gate, scale, bits, [out.get(name) for name in BLOCK_GRADS] if out else [])
    if rc:
        raise SFFNError("sffn_block_norm_backward", rc)
    return {name: t for name, t in zip(BLOCK_GRADS, got) if t is not None}


def _readable(t):
    """The rows t [T, D], or a copy of them where the calls do not take them as they lie: entries apart, or rows that start off 16 bytes."""
    as_it_is = t.stride(1) == 1 and t.data_ptr() % 16 == 0
    if t.shape[0] > 1:
        as_it_is = as_it_is and t.shape[1] <= t.stride(0) <= 1 << 31 and t.stride(0) * t.element_size() % 16 == 0
    return t if as_it_is else t.clone(memory_format=torch.contiguous_format)


class BlockNormFunction(torch.autograd.Function):
    """The pair as a node of torch's graph: ``h, n = BlockNormFunction.apply(y, resid, post_gain, pre_gain, gate, scale, eps, n_dtype)``,
    y and resid [..., D], at any strides, as gains and gate; n is None without pre_gain.  First derivatives only."""

    @staticmethod
    def forward(ctx, y, resid, post_gain=None, pre_gain=None, gate=None, scale=1.0, eps=1e-6, n_dtype=None):
        like = y if resid is None else resid
        D = like.shape[-1]
        rows = lambda t: None if t is None else _readable(t.reshape(-1, D))  # noqa: E731
        vector = lambda t: t if t is None or t.is_contiguous() and t.data_ptr() % 16 == 0 else t.clone(memory_format=torch.contiguous_format)  # noqa: E731
        post_gain, pre_gain = vector(post_gain), vector(pre_gain)
        if gate is None or gate.dim() == 1:
            g = vector(gate)
        else:
            g = gate.reshape(-1, gate.shape[-1])
            g = g.contiguous() if g.shape[1] == 1 else _readable(g)
        save = any(ctx.needs_input_grad)
        ry, rx = rows(y), rows(resid)
        h, n, stats = block_norm_forward(ry, rx, post_gain, pre_gain, g, scale=scale, eps=eps, save=save, n_dtype=n_dtype)
        if y is None and h.data_ptr() == resid.data_ptr():
            h = h.clone()  # an output of a node is not its input
        if save:
            ctx.save_for_backward(ry, h, stats, post_gain, pre_gain, g)
            ctx.scale, ctx.shape, ctx.gate_shape, ctx.has_resid, ctx.n_type = scale, like.shape, None if gate is None else gate.shape, resid is not None, n_dtype
        ctx.set_materialize_grads(False)
        return h.view(like.shape), None if n is None else n.view(like.shape)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh, dn):
        if dh is None and dn is None:
            return (None,) * 8
        y, h, stats, post_gain, pre_gain, gate = ctx.saved_tensors

        rows = lambda t: None if t is None else _readable(t.reshape(h.shape))  # noqa: E731
        wanted = dict(zip(("dy", "dresid", "dpost_gain", "dpre_gain", "dgate"), ctx.needs_input_grad))
        got = block_norm_backward(rows(dh), rows(dn), y, h, stats, post_gain, pre_gain, gate, scale=ctx.scale, need=[k for k, w in wanted.items() if w])
        for name, shape in (("dy", ctx.shape), ("dresid", ctx.shape), ("dgate", ctx.gate_shape)):
            if name in got:
                got[name] = got[name].view(shape)
        return (*[got.get(name) for name in BLOCK_GRADS], None, None, None)
