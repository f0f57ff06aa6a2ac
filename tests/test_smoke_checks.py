"""What the smoke run checks of the block's norms and of Muon, on the CPU: formulas in 32 bits pass, and each of them with a mistake does not."""
from types import SimpleNamespace

import pytest
import torch

import block_reference
import muon_reference

from __graft_entry__ import check_block_and_muon


def forward(y, resid, post_gain, pre_gain, gate, scale, eps=1e-6):
    out, _ = block_reference.forward(y, resid, post_gain, pre_gain, gate, scale, eps)
    return out["h"].to(resid.dtype), out["n"].to(resid.dtype), out["stats"].float()


def backward(dh, dn, y, h, stats, post_gain, pre_gain, gate, scale):
    out, _ = block_reference.backward(dh, dn, y, h, stats, post_gain, pre_gain, gate, scale)
    return {k: t.to(h.dtype if k in ("dy", "dresid") else torch.float32) for k, t in out.items()}


def step(params, grads, states, lr, momentum, weight_decay, scale):
    p, m = muon_reference.step(params[0], grads[0], states[0]["m"], None, lr=lr, momentum=momentum, nesterov=True, weight_decay=weight_decay, scale=scale)
    params[0].copy_(p)
    states[0]["m"].copy_(m)


def library(**over):
    m = dict(block_norm_forward=forward, block_norm_backward=backward, orthogonalize=lambda u: muon_reference.orthogonal(u).float(), muon_step=step,
             muon_state=lambda p: dict(m=torch.zeros_like(p)), training_status=lambda dev: 0)
    return SimpleNamespace(**{**m, **over})


def test_formulas_pass():
    check_block_and_muon(library(), "cpu")


def gradient(name, factor):
    def call(*args, **how):
        got = backward(*args, **how)
        got[name] = got[name] * factor
        return got
    return dict(block_norm_backward=call)


@pytest.mark.parametrize("over", [
    *[gradient(name, 1.02) for name in ("dy", "dresid", "dpost_gain", "dpre_gain", "dgate")],
    dict(block_norm_forward=lambda *a, **k: forward(*a, **k, eps=0.1)),
    dict(orthogonalize=lambda u: muon_reference.orthogonal(u, steps=4).float()),
    dict(orthogonalize=lambda u: muon_reference.orthogonal(u.bfloat16()).float()),
    dict(muon_step=lambda *a, **k: step(*a, **{**k, "weight_decay": 0.0})),
    dict(muon_step=lambda *a, **k: step(*a, **{**k, "lr": k["lr"] * 1.001})),
    dict(muon_step=lambda *a, **k: step(*a, **{**k, "momentum": 0.91})),
    dict(training_status=lambda dev: 5)])
def test_mistakes_do_not(over):
    with pytest.raises(AssertionError):
        check_block_and_muon(library(**over), "cpu")
