"""A model in 64 bits of Newton-Schulz steps whose products take operands of a few bits, and how far results in 32 bits may be off: what is left of
the roundings where tests of whole matrices, norm by norm, would not tell eleven bits from eight."""
import torch

from muon_reference import COEFFICIENTS

FP16, BF16 = 11, 8  # bits of an operand


def rounded(x, bits):
    """To the nearest of so many bits, at any exponent."""
    m, e = torch.frexp(x)
    return torch.ldexp(torch.round(m * 2.0 ** bits) / 2.0 ** bits, e)


class Held:
    """A symmetric matrix as its diagonal in 64 bits and the rest in a few."""

    def __init__(self, m, bits):
        self.d = m.diagonal().clone()
        self.rest = rounded(m - torch.diag(self.d), bits)

    def whole(self):
        return self.rest + torch.diag(self.d)

    def __matmul__(self, other):
        return self.rest @ other.rest + self.d[:, None] * other.rest + self.rest * other.d + torch.diag(self.d * other.d)


def modelled(u, bits, steps=5, coefficients=COEFFICIENTS, eps=1e-7, company=1):
    """Steps one at a time, or two in company: with B = b A + c A^2, D = a A + A B, A' = a D + D B and B' of A', R = a B' + a B + B B' and
    X'' = a^2 X + R X.  X itself and all sums in 64 bits.  The polynomial's diagonal multiplies what its rest does, X's operand, but for the
    steps behind which small singular values grow by four at most: X itself there."""
    a, b, c = coefficients
    x = u.double()
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    x = x / (x.norm() + eps)
    k = 0
    while k < steps:
        many = min(company, steps - k)
        hi = rounded(x, bits)
        A = Held(hi @ hi.T, bits)
        R = Held(b * A.whole() + c * (A @ A), bits)
        if many == 2:
            B = R
            D = Held(a * A.whole() + A @ B, bits)
            A = Held(a * D.whole() + D @ B, bits)
            second = Held(b * A.whole() + c * (A @ A), bits)
            R = Held(a * second.whole() + a * B.whole() + B @ second, bits)
        k += many
        x = a ** many * x + R.rest @ hi + R.d[:, None] * (x if abs(a) ** (steps - k) <= 4 else hi)
    return x.T if tall else x


def room16(u, want, dtype, steps=5):
    """How far an O of full rank from one fp16 term an operand may be off, relative to its norm: what the model is off with as many bits, and a
    quarter, whichever way of taking the steps leaves more (two in company make nothing good of what the first one leaves).  Roundings
    are independent, so the norm of what they leave varies by a few percent from draw to draw, and doubles with every bit less.  Own roundings
    come on top."""
    size = want.norm()
    most = max((modelled(u, FP16, steps, company=n) - want).norm().item() for n in (1, 2))
    return (1.25 * most + (want.to(dtype).double() - want).norm().item()) / size.item()


def room32(size, steps, a=COEFFICIENTS[0]):
    """The same of two terms an operand, whatever the rank, relative to O's norm `size`.

    A run of eight K blocks is 32 additions onto an accumulator that truncate, half a unit each, and where one entry dominates the sum is as large as
    it gets from the first on: products are off by as much as 32 2^-24.  Within X's own space a step takes A by b + c (2.8), A^2 by c (2.1) and
    the last product by 2.8, and the slopes of the polynomial at most double what is left.  What turns A's vectors outward is taken by what
    the polynomial of all steps in company, three at most, has at zero: a^3, of five products (A, B, D, A', R).  What lies outside on either
    side is the rounding of X, 2^-23 of an entry at most and 0.6 of that on the average, and grows by a in every step."""
    run = 32 * 2.0 ** -24
    return 2 * 7.7 * run + (5 * a ** min(steps, 3) * run + steps * a ** steps * 0.6 * 2.0 ** -23) / size
