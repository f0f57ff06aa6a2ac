"""What is asked of the fp32 training calls on the tensor cores, norm by norm, and their products in bf16 terms with exact sums, so that it can
be seen on a CPU what a product too few would do."""
import torch

import training_reference as ref

# On the tensor cores, of which shapes with hidden widths of every remainder, tiles that are cut and tiles that are whole.
SHAPES = [(700, 328, 900), (300, 2048, 2045), (40, 2048, 4097), (520, 1032, 4099), (1100, 1024, 2600)]
ACTS = [("sqrelu", "silu"), ("relu", None), ("rsplus", "relu")]

# The norm of an output's error over the output's norm.  Sums: a run of 128 k ends with eight MMAs on a full-size accumulator, which is truncated
# by up to 5e-8 each time four of them are added, 1e-7; what six products leave out is 2^-26 and less, the additions of runs round by
# 2^-25 each, at random: 2e-7 in all.  h, dz and du carry two to three such errors (a square doubles one) and some units of 2^-24 of their
# activations, 6e-7; a second product adds its own.  Twice that is allowed.  With three products the terms are 2^-17 and 2^-16 off.
LIMIT = 1.5e-6


def error(got, want):
    got, want = got.detach().cpu().double(), want.double()
    return float((got - want).norm() / want.norm())


def terms(t):
    out, rest = [], t.float()
    for _ in range(3):
        out.append(rest.bfloat16())
        rest = rest - out[-1].float()
    return [o.double() for o in out]


def product(a, b, six=True):
    """a b in terms, sums in 64 bits, rounded to fp32 once; three products instead of six: those without a third term, but a1 b1."""
    a, b = terms(a), terms(b)
    pairs = [(0, 0), (0, 1), (1, 0)] + ([(1, 1), (0, 2), (2, 0)] if six else [])
    return sum(a[i] @ b[j] for i, j in pairs)


def forward(x, W_g, b_g, W_up, W_down, a, a_up, six=True):
    z, u = product(x, W_g.T, six) + b_g.double(), product(x, W_up.T, six)
    h = (ref.act(a, z)[0] * ref.act(a_up, u)[0]).float()
    return dict(y=product(h, W_down, six).float(), z=z.float(), u=u.float())


def backward(dy, x, z, u, W_g, W_up, W_down, a, a_up, six=True):
    (av, da), (bv, db) = ref.act(a, z.double()), ref.act(a_up, u.double())
    dh = product(dy, W_down.T, six)
    dz, du, h = ((t).float() for t in (dh * bv * da, dh * av * db, av * bv))
    return dict(dx=(product(dz, W_g, six) + product(du, W_up, six)).float(), dW_g=product(dz.T, x, six).float(), dW_up=product(du.T, x, six).float(),
                dW_down=product(h.T, dy, six).float(), db_g=dz.double().sum(0).float())


def make(T, D, H, device="cpu", seed=0):
    g = torch.Generator()
    g.manual_seed(seed + 1000 * T + D + H)
    rnd = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).to(device)  # noqa: E731
    t = dict(x=rnd(T, D), W_g=rnd(H, D, std=D ** -0.5), b_g=rnd(H) - 0.8, W_up=rnd(H, D, std=D ** -0.5), W_down=rnd(H, D, std=D ** -0.5), dy=rnd(T, D))
    ld = (H + 7) // 8 * 8
    t["z"], t["u"] = (rnd(T, ld)[:, :H] for _ in range(2))
    return t


FORWARD = ("x", "W_g", "b_g", "W_up", "W_down")
BACKWARD = ("dy", "x", "z", "u", "W_g", "W_up", "W_down")
