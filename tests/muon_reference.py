"""The orthogonalised update and the Muon step in 64 bits, and how far the library's may be off, norm by norm."""
import math

import torch

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def orthogonal(u, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    triples = coefficients if hasattr(coefficients[0], "__len__") else [coefficients] * steps
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (x.norm() + eps)
    for a, b, c in triples:
        p = x @ x.T
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.T if tall else x


def step(p, g, m, master, *, lr, momentum, nesterov, weight_decay, scale, clip=1.0, **how):
    """(p, m) after a step; p before it is rounded."""
    g = g.double() * clip
    m = momentum * m.double() + (1 - momentum) * g
    u = (1 - momentum) * g + momentum * m if nesterov else m
    o = orthogonal(u, **how)
    return (p if master is None else master).double() * (1 - lr * weight_decay) - lr * scale * o, m


def room(bits, steps, a, size):
    """How far O may be off, relative to its norm `size`.

    Products: in a step P and Q are rounded once each, by 2^-11 of an entry in one fp16 term (2^-22 in two), 0.4 of that on the average
    over mantissas, and enter through b (4.8) and Q's values (2.8); steps' errors are independent, and slopes of the polynomial between
    them at most double what is left: 2 sqrt(steps) 5.6 0.4 2^-11 = 5e-3 in five steps.  In two terms the accumulators' truncation comes on
    top, 4e-7 of P in a run of eight K blocks, 4.8 times in every step: 1e-5 in five.
    What is amplified: a X is held in two terms, 2^-23 of an entry off at most, and 0.6 of that on the average in each step, and what lies
    outside X's own space grows by a in every step from then on: a^steps 0.6 2^-23 of the first X's norm, 1, each."""
    if bits == 16:
        products = 2 * math.sqrt(steps) * 5.6 * 0.4 * 2.0 ** -11
    else:
        products = 2 * math.sqrt(steps) * 5.6 * 0.4 * 2.0 ** -22 + steps * 4.8 * 4e-7
    return products + steps * max(a, 1.0) ** steps * 0.6 * 2.0 ** -23 / max(size, 1e-30)


def close(got, want, bits, steps=5, a=COEFFICIENTS[0]):
    """got's own rounding, and the room of its products."""
    assert got.shape == want.shape
    if want.numel() == 0:
        return
    size = want.norm().item()
    error = (got.double() - want).norm().item() / max(size, 1e-300)
    limit = torch.finfo(got.dtype).eps / 2 + room(bits, steps, a, size)
    assert error <= limit, (error, limit, tuple(got.shape))
