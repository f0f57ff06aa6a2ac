"""The norms around a block and their gradients in 64 bits, each with the size of the terms that make it up: what the roundings of a
computation in 32 bits are relative to."""
import torch

U32 = 2.0 ** -24


def unit(dtype):
    """Half a step of a type, relative."""
    return torch.finfo(dtype).eps / 2


def wide(t):
    return None if t is None else t.double()


def forward(y, resid, post_gain, pre_gain, gate, scale, eps):
    """h, n, stats and the sizes of h's and n's terms."""
    y, resid, post_gain, pre_gain, gate = map(wide, (y, resid, post_gain, pre_gain, gate))
    like = y if resid is None else resid
    h = torch.zeros_like(like) if resid is None else resid.clone()
    size_h, r = h.abs(), torch.zeros(like.shape[0], dtype=torch.float64, device=like.device)
    if y is not None:
        v = y
        if post_gain is not None:
            r = (y.square().mean(1) + eps).rsqrt()
            v = y * r[:, None] * post_gain
        v = scale * v if gate is None else scale * gate * v
        h, size_h = h + v, size_h + v.abs()
    rho = torch.zeros_like(r)
    n = size_n = None
    if pre_gain is not None:
        rho = (h.square().mean(1) + eps).rsqrt()
        n = h * rho[:, None] * pre_gain
        # h's own error, and through the norm that of its other entries
        size_n = (size_h + h.abs() * rho[:, None] ** 2 * (h.abs() * size_h).mean(1, keepdim=True)) * rho[:, None] * pre_gain.abs()
    return dict(h=h, n=n, stats=torch.stack([r, rho])), dict(h=size_h, n=size_n)


def backward(dh, dn, y, h, stats, post_gain, pre_gain, gate, scale):
    """Every gradient, and the size of its terms."""
    dh, dn, y, h, stats, post_gain, pre_gain, gate = map(wide, (dh, dn, y, h, stats, post_gain, pre_gain, gate))
    D = h.shape[1]
    g = torch.zeros_like(h) if dh is None else dh.clone()
    size = g.abs()
    out, sizes = {}, {}
    if dn is not None:
        rho = stats[1][:, None]
        t = pre_gain * dn
        g = g + rho * t - h * rho ** 3 * ((t * h).sum(1, keepdim=True) / D)
        size = size + rho * t.abs() + h.abs() * rho ** 3 * ((t * h).abs().sum(1, keepdim=True) / D)
    out["dresid"], sizes["dresid"] = g, size
    if pre_gain is not None:
        term = torch.zeros_like(h) if dn is None else dn * h * stats[1][:, None]
        out["dpre_gain"], sizes["dpre_gain"] = term.sum(0), term.abs().sum(0)
    if y is None:
        return out, sizes
    r = stats[0][:, None] if post_gain is not None else torch.ones_like(stats[0][:, None])
    gain = torch.ones(D, dtype=torch.float64, device=h.device) if post_gain is None else post_gain
    open_ = torch.ones(1, dtype=torch.float64, device=h.device) if gate is None else gate
    w = scale * gain * open_
    if post_gain is None:
        out["dy"], sizes["dy"] = w * g, w.abs() * size
    else:
        out["dy"] = r * w * g - y * r ** 3 * ((w * y * g).sum(1, keepdim=True) / D)
        sizes["dy"] = r * w.abs() * size + y.abs() * r ** 3 * ((w * y).abs() * size).sum(1, keepdim=True) / D
        out["dpost_gain"] = (scale * open_ * g * y * r).sum(0)
        sizes["dpost_gain"] = (scale * open_ * y * r).abs().mul(size).sum(0)
    if gate is not None:
        full, big = scale * g * gain * y * r, (scale * gain * y * r).abs() * size
        if gate.dim() == 1:
            full, big = full.sum(0), big.sum(0)
        elif gate.shape[1] == 1:
            full, big = full.sum(1, keepdim=True), big.sum(1, keepdim=True)
        out["dgate"], sizes["dgate"] = full, big
    return out, sizes


# Steps of 2^-24 that a value may be off, relative to the size of its terms.  A row's sum: eight products and as many sums a piece, up to
# four pieces, five exchanges in a warp and five among warps are at most 45 roundings on the way; the square root doubles none of
# them (it halves them), rsqrtf adds two units, the factors and the last sum ten.
ROW = 64
# A column's sum adds up to 64 roundings in a CTA for every 64 rows that it meets, and 64 more over the lines.
def column(T):
    return ROW + 64 + T // 16


def close(name, got, want, size, steps):
    """got within its own rounding and `steps` of 2^-24 of the terms' size."""
    assert got.shape == want.shape, name
    room = unit(got.dtype) * want.abs() + (steps * U32) * size * (1 + unit(got.dtype)) + 1e-300
    worst = ((got.double() - want).abs() / room).max().item() if got.numel() else 0.0
    assert worst <= 1.0, (name, worst)
