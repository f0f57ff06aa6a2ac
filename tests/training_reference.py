"""Plain 64-bit forms of the training operators, and the rounding bounds that their tests use."""
import torch

U16 = 2.0 ** -8    # half a unit in the last place of bf16, relative: 8 significant bits
U32 = 2.0 ** -24   # of fp32


def act(name, t):
    """Value and slope of an activation (slope 0 at 0 for those that are 0 below it)."""
    if name in (None, "none"):
        return t, torch.ones_like(t)
    if name == "silu":
        s = torch.sigmoid(t)
        return t * s, s * (1 + t * (1 - s))
    on = (t > 0).to(t.dtype)
    p = t * on
    if name == "relu":
        return p, on
    if name == "sqrelu":
        return p * p, 2 * p
    s = torch.sigmoid(p)
    return p * s, on * s * (1 + p * (1 - s))


def wide(*tensors):
    return [None if t is None else t.detach().cpu().double() for t in tensors]


def forward(x, W_g, b_g, W_up, W_down, a, a_up):
    x, W_g, b_g, W_up, W_down = wide(x, W_g, b_g, W_up, W_down)
    z, u = x @ W_g.T, x @ W_up.T
    if b_g is not None:
        z = z + b_g
    h = act(a, z)[0] * act(a_up, u)[0]
    return dict(y=h @ W_down, z=z, u=u)


def backward(dy, x, z, u, W_g, W_up, W_down, a, a_up):
    dy, x, z, u, W_g, W_up, W_down = wide(dy, x, z, u, W_g, W_up, W_down)
    (av, da), (bv, db) = act(a, z), act(a_up, u)
    dh = dy @ W_down.T
    dz, du, h = dh * bv * da, dh * av * db, av * bv
    return dict(dx=dz @ W_g + du @ W_up, dW_g=dz.T @ x, dW_up=du.T @ x, dW_down=h.T @ dy, db_g=dz.sum(0))


def forward_bounds(x, W_g, b_g, W_up, W_down, a, a_up, bf16):
    """How far each entry may be off.  A sum of K products in fp32, in any order, with up to two rounding units a step, is within
    (K + 8) 2 U32 of the sum of its terms' magnitudes S.  h = A A_3 then carries the relative error of its factors: |A'| dz A_3 +
    A A_3' du, some units of its own, and with bf16 storage one rounding; outputs are rounded once."""
    x, W_g, b_g, W_up, W_down = wide(x, W_g, b_g, W_up, W_down)
    out = U16 if bf16 else U32
    D, H = x.shape[1], W_g.shape[0]
    zb = torch.zeros(H, dtype=torch.float64) if b_g is None else b_g
    z, u = x @ W_g.T + zb, x @ W_up.T
    ez = (D + 8) * 2 * U32 * (x.abs() @ W_g.abs().T + zb.abs())
    eu = (D + 8) * 2 * U32 * (x.abs() @ W_up.abs().T)
    (av, da), (bv, db) = act(a, z), act(a_up, u)
    # an activation's slope is at most 1.1 between z and where an error of ez puts it, but for the square
    sa = 2 * (z.abs() + ez) if a == "sqrelu" else torch.full_like(z, 1.1)
    sb = 2 * (u.abs() + eu) if a_up == "sqrelu" else torch.full_like(u, 1.1)
    h = (av * bv).abs()
    eh = sa * ez * bv.abs() + sb * eu * av.abs() + sa * sb * ez * eu + h * (64 * U32 if not bf16 else U16 + 2 ** -18)
    y = (av * bv) @ W_down
    ey = eh @ W_down.abs() + (H + 8) * 2 * U32 * ((h + eh) @ W_down.abs())
    # 2^-133: half the smallest bf16 (and more than half the smallest fp32)
    return dict(z=ez + out * (z.abs() + ez) + 2.0 ** -133, u=eu + out * (u.abs() + eu) + 2.0 ** -133, y=ey + out * (y.abs() + ey) + 2.0 ** -133)


def backward_bounds(dy, x, z, u, W_g, W_up, W_down, a, a_up, bf16):
    """The same for the gradients: dh is a sum over D, its products with slopes and values carry a few units and one rounding to
    bf16 before they enter the next products; db_g sums them before that."""
    dy, x, z, u, W_g, W_up, W_down = wide(dy, x, z, u, W_g, W_up, W_down)
    out = U16 if bf16 else U32
    T, D, H = x.shape[0], x.shape[1], W_g.shape[0]
    (av, da), (bv, db) = act(a, z), act(a_up, u)
    dh = dy @ W_down.T
    edh = (D + 8) * 2 * U32 * (dy.abs() @ W_down.abs().T)
    units = 2 ** -17 if bf16 else 64 * U32  # value and slope of an activation
    hidden = {}
    for name, f in (("dz", bv * da), ("du", av * db)):
        v = dh * f
        # a slope's own error is relative to the terms it is made of, at most 1.3
        hidden[name] = (v, edh * f.abs() + units * (dh.abs() + edh) * (f.abs() + 1.3 * (bv if name == "dz" else av).abs()))
    h = av * bv
    hidden["h"] = (h, units * h.abs())
    stored = {k: (v, e + (U16 * (v.abs() + e) if bf16 else 0)) for k, (v, e) in hidden.items()}

    def product(pairs, K):
        total, err, ref = 0, 0, 0
        for (v, e), w, left in pairs:
            s = (v.abs() + e).T @ w.abs() if left else (v.abs() + e) @ w.abs()
            total = total + s
            err = err + (e.T @ w.abs() if left else e @ w.abs())
            ref = ref + (v.T @ w if left else v @ w)
        err = err + (K + 8) * 2 * U32 * total
        return err + out * (ref.abs() + err) + 2.0 ** -133

    dz, edz = hidden["dz"]
    edb = edz.sum(0) + (T + 8) * 2 * U32 * (dz.abs() + edz).sum(0)
    return dict(dx=product([(stored["dz"], W_g, False), (stored["du"], W_up, False)], 2 * H), dW_g=product([(stored["dz"], x, True)], T),
                dW_up=product([(stored["du"], x, True)], T), dW_down=product([(stored["h"], dy, True)], T), db_g=edb + 2.0 ** -133)


def assert_within(got, ref, bounds, what=""):
    for k, r in ref.items():
        g = got[k].detach().cpu().double()
        assert g.shape == r.shape, (what, k, g.shape, r.shape)
        assert torch.isfinite(g).all(), (what, k)
        off = (g - r).abs() - bounds[k]
        assert off.numel() == 0 or off.max() <= 0, f"{what} {k}: {int((off > 0).sum())} entries beyond the bound, by up to {float(off.max()):.3e} at {divmod(int(off.argmax()), r.shape[-1])}"


def adamw(p, g, m, v, step, lr, betas, eps, weight_decay, scale=1.0):
    """One step in 64 bits: (p, m, v)."""
    p, g, m, v = wide(p, g, m, v)
    g = g * scale
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    p = p * (1 - lr * weight_decay) - lr * (m / (1 - betas[0] ** step)) / ((v / (1 - betas[1] ** step)).sqrt() + eps)
    return p, m, v


def decode(codes, scale, levels, power, group=256):
    """fp64 values of codes."""
    c = codes.detach().cpu().double().reshape(-1)
    s = scale.detach().cpu().double().repeat_interleave(group)[:c.numel()]
    return (c.sign() * (c.abs() / levels) ** power * s).view(codes.shape)
