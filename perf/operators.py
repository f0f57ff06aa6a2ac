"""The training operators of this library as measurable cases: the gated FFN with its backward pass, the norm of a model's
gradients, and an AdamW step over a list of tensors.

Every case computes one pass of one operator.  `run` does so in elementary torch operations in 32 bits, or, where `own` is
true, through the library's entry points; `exact` states the same definitions in 64 bits.
"""
import math
import statistics

import torch

own = False

DEV = "cuda:0"
BETAS, EPS = (0.9, 0.999), 1e-8
BLOCK = 256          # consecutive entries of a tensor that share the scales of their 8-bit states
TINY = 2.0 ** -100   # a block whose largest value is below this is stored as zeros
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ESZ = {"f32": 4, "bf16": 2}


def ffn(op, dtype, T, D, H, act="relu", act_up="", s=0.9, **more):
    """op: "forward" or "backward" of y = (A(x W_g^T + b_g) . A_3(x W_up^T)) W_down over T tokens.  s: share of neurons that do
    not fire.  act_up: activation on the up projection ("" = none)."""
    return dict(op=op, dtype=dtype, T=T, D=D, H=H, act=act, act_up=act_up, s=s, **more)


def model(op, dtype, layers, D, H, bits=32, master=False, clip=False, step=100, **more):
    """op: "norm" or "adamw", over the three matrices and the gate bias of each of `layers` FFNs.  bits: of the two moments.
    master: bf16 matrices with a copy in 32 bits that takes the steps.  clip: the gradients are scaled by their norm."""
    return dict(op=op, dtype=dtype, layers=layers, D=D, H=H, bits=bits, master=master, clip=clip, step=step, **more)


def listed():
    return [
        # the smallest model of the benchmark, its 64 tokens: launches and latency
        ffn("forward", "f32", 64, 256, 1024, name="forward_small_f32"),
        # a ragged micro-batch under double activation, a 4096-wide model
        ffn("forward", "bf16", 1000, 4096, 14336, act="sqrelu", act_up="silu", name="forward_bf16"),
        # a whole batch of sequences through the same model
        ffn("forward", "bf16", 8192, 4096, 14336, name="forward_large_bf16"),
        # the backward pass of the smallest model
        ffn("backward", "f32", 64, 256, 1024, name="backward_small_f32"),
        # a handful of tokens (online fine-tuning): the weights' bytes and their gradients' count, not the products
        ffn("backward", "bf16", 5, 4096, 14336, name="backward_few_bf16"),
        # the micro-batch of a training step
        ffn("backward", "bf16", 4096, 4096, 14336, act="rsplus", name="backward_bf16"),
        # the paper's shape, a hidden width that no tile divides, in full precision
        ffn("backward", "f32", 500, 3840, 14230, act="sqrelu", name="backward_ragged_f32"),
        # gradients of the smallest model: latency
        model("norm", "f32", 1, 256, 1024, name="norm_small_f32"),
        # gradients of four layers of a 4096-wide model
        model("norm", "bf16", 4, 4096, 14336, name="norm_bf16"),
        # sixteen layers of the smallest model: many tensors, few bytes each
        model("adamw", "f32", 16, 256, 1024, name="adamw_many_f32"),
        # a layer of the paper's shape: bf16 weights, a copy in 32 bits, moments in 32 bits, clipped gradients
        model("adamw", "bf16", 1, 3840, 14230, master=True, clip=True, name="adamw_master_bf16"),
        # a layer of the widest model: bf16 weights, moments in 8 bits, read back for a checkpoint after the step
        model("adamw", "bf16", 1, 8192, 28672, bits=8, clip=True, name="adamw_8bit_bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_once(rng):
    op = rng.choice(["forward", "forward", "backward", "backward", "norm", "adamw", "adamw"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    D = max(256, round(_log_uniform(rng, 256, 8192) / 8) * 8)
    H = min(28672, round(D * rng.uniform(2.0, 4.0)))
    if rng.random() < 0.5:
        H = H // 64 * 64
    if op in ("forward", "backward"):
        return ffn(op, dtype, round(_log_uniform(rng, 1, 8192)), D, H, act=rng.choice(["relu", "sqrelu", "rsplus", "silu"]),
                   act_up=rng.choice(["", "", "relu", "silu"]), s=round(rng.uniform(0.5, 0.95), 3))
    if op == "norm":
        return model(op, dtype, rng.randint(1, 16), D, H)
    return model(op, dtype, rng.randint(1, 16), D, H, bits=rng.choice([8, 32]), master=dtype == "bf16" and rng.random() < 0.5,
                 clip=rng.random() < 0.5, step=rng.randint(1, 20000))


def _price(c):
    w = work(c)
    rate = 6e13 if c["dtype"] == "f32" else 1.4e15
    return w["bytes"] / 6.5e12 + w["flops"] / rate


def draw(rng):
    every = listed()
    most = {op: max(_price(c) for c in every if c["op"] == op) for op in ("forward", "backward", "norm", "adamw")}
    while True:
        c = _draw_once(rng)
        if _price(c) <= most[c["op"]]:
            return c


def _rows(T, H, dtype):
    """A [T, H] matrix whose rows are a multiple of 16 bytes apart, as the entry points take it."""
    return torch.empty((T, (H + 7) // 8 * 8), dtype=dtype, device=DEV)[:, :H]


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(shape, std, dtype, gen):
    return torch.randn(shape, generator=gen, device=DEV).mul_(std).to(dtype)


def _prepare_ffn(c, seed):
    gen, dtype = _gen(seed), DTYPES[c["dtype"]]
    T, D, H = c["T"], c["D"], c["H"]
    st = dict(op=c["op"], act=c["act"], act_up=c["act_up"] or None)
    st["x"] = _normal((T, D), 1.0, dtype, gen)
    st["W_g"], st["W_up"], st["W_down"] = (_normal((H, D), D ** -0.5, dtype, gen) for _ in range(3))
    b = -statistics.NormalDist().inv_cdf(c["s"])
    st["b_g"] = b + 0.1 * torch.randn(H, generator=gen, device=DEV)
    if c["op"] == "backward":  # what the forward pass saved, and the gradient of a mean over the tokens
        for name, shift in (("z", b), ("u", 0.0)):
            st[name] = _rows(T, H, dtype)
            st[name].copy_(torch.randn((T, H), generator=gen, device=DEV) + shift)
        st["dy"] = _normal((T, D), 1.0 / T, dtype, gen)
    return st


def _shapes(c):
    return [s for _ in range(c["layers"]) for s in [(c["H"], c["D"])] * 3 + [(c["H"],)]]


def _arena(c, kind, dtype):
    """One buffer for all tensors of a kind ("matrices", "biases"), each at a multiple of BLOCK entries, and its slices in order."""
    shapes = [s for s in _shapes(c) if (len(s) == 2) == (kind == "matrices")]
    room = (math.prod(shapes[0]) + BLOCK - 1) // BLOCK * BLOCK
    buf = torch.zeros(room * len(shapes), dtype=dtype, device=DEV)
    return buf, [buf[i * room:i * room + math.prod(s)].view(s) for i, s in enumerate(shapes)]


def _in_order(c, matrices, biases):
    """The slices of both kinds as the model lists its tensors: three matrices and a bias a layer."""
    return [t for i in range(c["layers"]) for t in (*matrices[3 * i:3 * i + 3], biases[i])]


def _gradients(c, gen):
    """Gradients of a batch: noise, and nothing at all for one neuron in five, which no token fired."""
    grads = []
    for shape in _shapes(c):
        g = torch.randn(shape, generator=gen, device=DEV).mul_(1e-4)
        fired = torch.rand(shape[0], generator=gen, device=DEV) >= 0.2
        grads.append((g * fired[:, None] if len(shape) == 2 else g * fired).to(DTYPES[c["dtype"]] if len(shape) == 2 else torch.float32))
    return grads


def _prepare_model(c, seed):
    gen = _gen(seed)
    st = dict(op=c["op"], grads=_gradients(c, gen))
    if c["op"] == "norm":
        return st
    st.update(bits=c["bits"], step=c["step"], lr=3e-4, weight_decay=[0.1, 0.1, 0.1, 0.0] * c["layers"])
    st["max_norm"] = 1.0 if c["clip"] else None
    st["grad_norm"] = 1.0 + torch.rand((), generator=gen, device=DEV) if c["clip"] else None
    q = c["bits"] == 8
    types = dict(m=torch.int8, v=torch.uint8) if q else dict(m=torch.float32, v=torch.float32)
    if q:  # where the moments are read back to
        types.update(m_value=torch.float32, v_value=torch.float32)
    if c["master"]:
        types.update(master=torch.float32)
    whole, parts = dict(matrices={}, biases={}), {}
    for key, dtype in dict(types, p=None).items():
        for kind in whole:
            t = dtype or (DTYPES[c["dtype"]] if kind == "matrices" else torch.float32)
            if key != "master" or kind == "matrices":
                whole[kind][key], parts[kind] = _arena(c, kind, t)
            else:
                parts[kind] = [None] * c["layers"]
        parts[key] = _in_order(c, parts["matrices"], parts["biases"])
    st.update(whole=whole, params=parts["p"], masters=parts.get("master") or [None] * len(parts["p"]), states=[])
    for i, (p, w) in enumerate(zip(st["params"], st["masters"])):
        start = torch.randn(p.shape, generator=gen, device=DEV).mul_(c["D"] ** -0.5)
        p.copy_(start)
        if w is not None:
            w.copy_(start)
        m, v = parts["m"][i], parts["v"][i]
        state = dict(m=m, v=v)
        if q:  # moments as a step leaves them: codes and a scale for every 256 entries
            m.copy_(torch.randn(p.shape, generator=gen, device=DEV).mul_(40.0).round_().clamp_(-127, 127))
            v.copy_(torch.randn(p.shape, generator=gen, device=DEV).mul_(40.0).add_(150.0).round_().clamp_(1, 255))
            scale = 1.0 + torch.rand((2, (p.numel() + BLOCK - 1) // BLOCK), generator=gen, device=DEV)
            state.update(m_scale=scale[0] * 1e-4, v_scale=scale[1] * 1e-7)
        else:
            m.copy_(torch.randn(p.shape, generator=gen, device=DEV).mul_(3e-5))
            v.copy_(torch.randn(p.shape, generator=gen, device=DEV).square_().mul_(1e-8))
        st["states"].append(state)
    if q:
        st["values"] = [dict(m=m, v=v) for m, v in zip(parts["m_value"], parts["v_value"])]
    return st


def prepare(c, seed):
    return _prepare_ffn(c, seed) if c["op"] in ("forward", "backward") else _prepare_model(c, seed)


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _act(name, z):
    if name is None:
        return z
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    p = z.clamp(min=0.0)
    return p if name == "relu" else p * p if name == "sqrelu" else p / (1.0 + torch.exp(-p))


def _slope(name, z):
    """The derivative of _act; 0 at 0 for the activations that are 0 below it."""
    if name is None:
        return torch.ones_like(z)
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "sqrelu":
        return 2.0 * z.clamp(min=0.0)
    s = 1.0 / (1.0 + torch.exp(-z))
    d = s * (1.0 + z * (1.0 - s))
    return d if name == "silu" else d * (z > 0)


def _forward(st):
    x, dtype = st["x"].float(), st["x"].dtype
    z = x @ st["W_g"].float().T + st["b_g"]
    u = x @ st["W_up"].float().T
    y = (_act(st["act"], z) * _act(st["act_up"], u)) @ st["W_down"].float()
    return dict(y=y.to(dtype), z=z.to(dtype), u=u.to(dtype))


def _backward(st):
    dy, x, z, u = (st[k].float() for k in ("dy", "x", "z", "u"))
    dtype = st["x"].dtype
    a, b = _act(st["act"], z), _act(st["act_up"], u)
    dh = dy @ st["W_down"].float().T
    dz, du = dh * b * _slope(st["act"], z), dh * a * _slope(st["act_up"], u)
    dx = dz @ st["W_g"].float() + du @ st["W_up"].float()
    return dict(dx=dx.to(dtype), dW_g=(dz.T @ x).to(dtype), dW_up=(du.T @ x).to(dtype), dW_down=((a * b).T @ dy).to(dtype), db_g=dz.sum(0))


def _norm(grads):
    return torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()


def _blocks(t):
    """The entries of t in rows of BLOCK, the last one filled up with zeros."""
    t, more = t.reshape(-1), -t.numel() % BLOCK
    return (torch.cat([t, t.new_zeros(more)]) if more else t).view(-1, BLOCK)


def _decode(state, shape):
    """m = s sign(c) (c / 127)^2, v = s (c / 255)^4."""
    n = math.prod(shape)
    cm, cv = _blocks(state["m"]).float(), _blocks(state["v"]).float()
    m = cm * cm.abs() * (state["m_scale"] * (1.0 / 127.0 ** 2))[:, None]
    v = (cv * cv).square() * (state["v_scale"] * (1.0 / 255.0 ** 4))[:, None]
    return m.view(-1)[:n].view(shape), v.view(-1)[:n].view(shape)


def _encode_one(t, top, edges):
    """Scales and codes of rows of BLOCK values t >= 0: the code is the number of edges at or below top t / scale."""
    s = t.amax(1)
    keep = s >= TINY
    q = t * torch.where(keep, s, torch.ones_like(s)).reciprocal()[:, None] * top
    code = torch.bucketize(q, edges, right=True) * keep[:, None]
    return torch.where(keep, s, torch.zeros_like(s)), code


def _encode(m, v, state):
    k = torch.arange(255, dtype=torch.float32, device=m.device)
    k = k * k + k + 0.25                                     # (code + 1/2)^2, exact in 32 bits
    n, mb, vb = m.numel(), _blocks(m), _blocks(v)
    state["m_scale"], code = _encode_one(mb.abs(), 127.0 ** 2, k[:127])
    state["m"].view(-1).copy_((code * mb.sign().to(torch.int64)).view(-1)[:n])
    state["v_scale"], code = _encode_one(vb, 255.0 ** 4, k.square())
    some = (vb > 0) & (state["v_scale"] > 0)[:, None]        # what is not zero stays so: it divides
    state["v"].view(-1).copy_(torch.where(some, code.clamp(min=1), code).view(-1)[:n])


def _adamw(st):
    b1, b2 = BETAS
    bc1, bc2 = 1.0 - b1 ** st["step"], 1.0 - b2 ** st["step"]
    lr, scale = st["lr"], None
    if st["max_norm"] is not None:
        norm = st["grad_norm"]
        scale = (torch.full_like(norm, st["max_norm"]) / (norm + 1e-6)).clamp(max=1.0)
    for i, (p, g, state, master, wd) in enumerate(zip(st["params"], st["grads"], st["states"], st["masters"], st["weight_decay"])):
        g = g.float()
        if scale is not None:
            g = g * scale
        m, v = _decode(state, p.shape) if st["bits"] == 8 else (state["m"], state["v"])
        m = m * b1 + g * (1.0 - b1)
        v = v * b2 + g * g * (1.0 - b2)
        w = (p if master is None else master).float()
        w = w * (1.0 - lr * wd) - m / (v.sqrt() * (1.0 / math.sqrt(bc2)) + EPS) * (lr / bc1)
        p.copy_(w)
        if master is not None:
            master.copy_(w)
        if st["bits"] == 8:
            _encode(m, v, state)
            m, v = _decode(state, p.shape)
            state = st["values"][i]
        state["m"].copy_(m)
        state["v"].copy_(v)
    return _answer(st)


def _answer(st):
    """All weights, copies in 32 bits and moments after the step; moments held in codes as the values that they stand for."""
    q = "_value" if st["bits"] == 8 else ""
    return {kind: {key: t[key + q if key in "mv" else key] for key in ("p", "m", "v", "master") if key in t} for kind, t in st["whole"].items()}


def run(st):
    if own:
        return _run_own(st)
    return {"forward": _forward, "backward": _backward, "norm": lambda s: _norm(s["grads"]), "adamw": _adamw}[st["op"]](st)


def _run_own(st):
    import paper_2609_31975_b200 as lib

    if st["op"] == "forward":
        y, z, u = lib.gated_ffn_forward(st["x"], st["W_g"], st["b_g"], st["W_up"], st["W_down"], st["act"], st["act_up"])
        return dict(y=y, z=z, u=u)
    if st["op"] == "backward":
        return lib.gated_ffn_backward(st["dy"], st["x"], st["z"], st["u"], st["W_g"], st["W_up"], st["W_down"], st["act"], st["act_up"])
    if st["op"] == "norm":
        return lib.grad_norm(st["grads"])
    lib.adamw_step(st["params"], st["grads"], st["states"], st["step"], lr=st["lr"], betas=BETAS, eps=EPS, weight_decay=st["weight_decay"],
                   masters=st["masters"], grad_norm=st["grad_norm"], max_norm=st["max_norm"])
    if st["bits"] == 8:
        lib.adamw_state_values(st["states"], out=st["values"])
    return _answer(st)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------


def work(c):
    e = ESZ[c["dtype"]]
    if c["op"] in ("forward", "backward"):
        T, D, H = c["T"], c["D"], c["H"]
        weights, tokens, hidden = 3 * H * D * e, T * D * e, T * H * e
        if c["op"] == "forward":  # x, weights, bias in; y, z, u out; three products
            return {"bytes": weights + 4 * H + 2 * tokens + 2 * hidden, "flops": 6.0 * T * D * H}
        # dy, x, z, u, weights in; dx, gradients out; six products
        return {"bytes": 2 * weights + 4 * H + 3 * tokens + 2 * hidden, "flops": 12.0 * T * D * H}
    mats, biases = 3.0 * c["layers"] * c["H"] * c["D"], float(c["layers"] * c["H"])
    if c["op"] == "norm":
        return {"bytes": mats * e + biases * 4, "flops": 2 * (mats + biases)}
    # p, m and v read and written, g read; with a copy in 32 bits that one is read and both are written; 8-bit moments also read back
    # as values in 32 bits
    weight = (2 + 8) if c["master"] else 2 * e
    state = 16 if c["bits"] == 32 else 4 * (1 + 4 / BLOCK) + (2 + 8 + 8 / BLOCK)
    return {"bytes": mats * (weight + e + state) + biases * (8 + 4 + state), "flops": 16 * (mats + biases)}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------


def _sigmoid64(t):
    return torch.special.expit(t)


def _pair64(name, t):
    """An activation and its derivative."""
    one = torch.ones_like(t)
    if name is None:
        return t, one
    pos = (t > 0).double()
    if name == "relu":
        return t * pos, pos
    if name == "sqrelu":
        return t * t * pos, 2 * t * pos
    s = _sigmoid64(t)
    value, slope = t * s, s + t * s * (1 - s)
    return (value, slope) if name == "silu" else (value * pos, slope * pos)


def _exact_ffn(c, seed):
    st = _prepare_ffn(c, seed)
    x, wg, wu, wd = (st[k].double() for k in ("x", "W_g", "W_up", "W_down"))
    if c["op"] == "forward":
        z = torch.einsum("td,hd->th", x, wg).add_(st["b_g"].double())
        u = torch.einsum("td,hd->th", x, wu)
        h = _pair64(st["act"], z)[0] * _pair64(st["act_up"], u)[0]
        return dict(y=torch.einsum("th,hd->td", h, wd), z=z, u=u)
    dy, z, u = (st[k].double() for k in ("dy", "z", "u"))
    (a, da), (b, db) = _pair64(st["act"], z), _pair64(st["act_up"], u)
    dh = torch.einsum("td,hd->th", dy, wd)
    gate, up = dh * da * b, dh * a * db
    return dict(dx=torch.einsum("th,hd->td", gate, wg) + torch.einsum("th,hd->td", up, wu), dW_g=torch.einsum("th,td->hd", gate, x),
                dW_up=torch.einsum("th,td->hd", up, x), dW_down=torch.einsum("th,td->hd", a * b, dy), db_g=gate.sum(dim=0))


def _values64(codes, scale, levels, power):
    n = codes.numel()
    s = scale.double().repeat_interleave(BLOCK)[:n]
    c = codes.reshape(-1).double() / levels
    return c.sign() * c.abs() ** power * s


def _through_codes64(t, levels, power, floor):
    """What values come back as after they were stored in codes."""
    n, out = t.numel(), torch.empty_like(t)
    edge = ((torch.arange(levels, dtype=torch.float64, device=t.device) + 0.5) / levels) ** power
    step = 1 << 24  # a piece at a time, whole blocks of it
    for i in range(0, n, step):
        part = t[i:i + step]
        size = part.numel()
        full = torch.zeros((size + BLOCK - 1) // BLOCK * BLOCK, dtype=torch.float64, device=t.device)
        full[:size] = part
        full = full.view(-1, BLOCK)
        s = full.abs().max(dim=1, keepdim=True).values
        s = s * (s >= TINY)
        r = torch.where(s > 0, full.abs() / s.clamp(min=TINY), 0.0)
        code = torch.searchsorted(edge, r, right=True).double()
        code = torch.where((r > 0) & (s > 0), code.clamp(min=floor), code)
        out[i:i + size] = (full.sign() * (code / levels) ** power * s).view(-1)[:size]
    return out


def _exact_adamw(c, seed):
    st = _prepare_model(c, seed)
    k, (b1, b2) = st["step"], BETAS
    scale = min(1.0, st["max_norm"] / (float(st["grad_norm"]) + 1e-6)) if c["clip"] else 1.0
    out, slices = dict(matrices={}, biases={}), {}
    for key in ("p", "m", "v"):
        for kind in out:
            out[kind][key], slices[kind] = _arena(c, kind, torch.float64)
        slices[key] = _in_order(c, slices["matrices"], slices["biases"])
    for i, p in enumerate(st["params"]):
        s, w = st["states"][i], st["masters"][i]
        g = st["grads"][i].reshape(-1).double() * scale
        if c["bits"] == 8:
            m, v = _values64(s["m"], s["m_scale"], 127, 2), _values64(s["v"], s["v_scale"], 255, 4)
        else:
            m, v = s["m"].reshape(-1).double(), s["v"].reshape(-1).double()
        m, v = m.lerp_(g, 1 - b1), v.mul_(b2).addcmul_(g, g, value=1 - b2)
        new = (p if w is None else w).reshape(-1).double() * (1 - st["lr"] * st["weight_decay"][i])
        new -= st["lr"] * (m / (1 - b1 ** k)) / ((v / (1 - b2 ** k)).sqrt() + EPS)
        if c["bits"] == 8:
            m, v = _through_codes64(m, 127, 2, 0), _through_codes64(v, 255, 4, 1)
        for key, t in (("p", new), ("m", m), ("v", v)):
            slices[key][i].copy_(t.view(p.shape))
    if c["master"]:
        out["matrices"]["master"] = out["matrices"]["p"]
    return out


def exact(c, seed):
    if c["op"] in ("forward", "backward"):
        return _exact_ffn(c, seed)
    if c["op"] == "norm":
        return sum(float((g.double() ** 2).sum()) for g in _gradients(c, _gen(seed))) ** 0.5 * torch.ones((), dtype=torch.float64, device=DEV)
    return _exact_adamw(c, seed)
