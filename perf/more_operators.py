"""The operators of a residual FFN block and of the Muon optimiser as measurable cases: an update made orthogonal by Newton-Schulz
products, a Muon step over a list of matrices, and the norms before and after a block with its gate and residual scale, forward
and backward.

Every case computes one pass of one operator.  `run` does so in elementary torch operations in 32 bits, or, where `own` is
true, through the library's entry points; `exact` states the same definitions in 64 bits.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ESZ = {"f32": 4, "bf16": 2}
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7
MOMENTUM, DECAY, MAX_NORM = 0.95, 0.1, 1.0
LR = dict(spectral=0.02, rms=1e-3)  # with either rule of the step's size
NORM_EPS = 1e-6
KEEP = 0.5  # residual scale of a block


def orthogonal(dtype, H, D, **more):
    """The update of one [H, D] matrix."""
    return dict(op="orthogonalize", dtype=dtype, H=H, D=D, **more)


def muon(dtype, layers, H, D, master=False, clip=False, nesterov=True, scale="spectral", **more):
    """A step over the three matrices of each of `layers` FFNs.  master: bf16 matrices with a copy in 32 bits that takes the step.
    clip: the gradients are scaled by their norm."""
    return dict(op="muon", dtype=dtype, layers=layers, H=H, D=D, master=master, clip=clip, nesterov=nesterov, scale=scale, **more)


def norms(op, T, D, y, stream, out, gate="none", post=True, pre=True, **more):
    """op: "forward" or "backward" of h = resid + scale gate N(y), n = N(h).  y, stream, out: types of the block's output, of the
    residual stream (resid and h), of n.  gate: one number a channel, a token or an entry, or none.  post, pre: which of the norms."""
    return dict(op=op, T=T, D=D, y=y, stream=stream, out=out, gate=gate, post=post, pre=pre, **more)


def listed():
    return [
        # a gate matrix of the benchmark's smallest model: latency of a chain of dependent products
        orthogonal("f32", 1024, 256, name="orthogonalize_small_f32"),
        # the paper's shape, a hidden width that no tile divides
        orthogonal("bf16", 14230, 3840, name="orthogonalize_ragged_bf16"),
        # a matrix of the widest model
        orthogonal("bf16", 28672, 8192, name="orthogonalize_large_bf16"),
        # sixteen layers of the smallest model, all in 32 bits: many matrices of one shape
        muon("f32", 16, 1024, 256, scale="rms", name="muon_many_f32"),
        # a layer of a 4096-wide model, weights in bf16 only
        muon("bf16", 1, 14336, 4096, name="muon_bf16"),
        # a layer of the paper's shape: copies in 32 bits, clipped gradients
        muon("bf16", 1, 14230, 3840, master=True, clip=True, scale="rms", name="muon_master_bf16"),
        # one decoded token: the FFN's fp32 output onto a bf16 stream, and the next block's norm
        norms("forward", 1, 4096, "f32", "bf16", "bf16", name="norms_decode"),
        # a ragged micro-batch, with a gate for every channel
        norms("forward", 1000, 4096, "bf16", "bf16", "bf16", gate="channel", name="norms_bf16"),
        # a whole batch of the widest model, stream in 32 bits
        norms("forward", 8192, 8192, "bf16", "f32", "bf16", gate="channel", name="norms_large"),
        # the smallest model's 64 tokens
        norms("backward", 64, 256, "f32", "f32", "f32", gate="channel", name="norms_backward_small_f32"),
        # the micro-batch of a training step
        norms("backward", 4096, 4096, "bf16", "bf16", "bf16", gate="channel", name="norms_backward_bf16"),
        # the paper's width, a gate for every token, stream in 32 bits
        norms("backward", 5000, 3840, "bf16", "f32", "bf16", gate="token", name="norms_backward_token_gate"),
    ]


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_once(rng):
    op = rng.choice(["orthogonalize", "orthogonalize", "muon", "muon", "forward", "forward", "backward", "backward"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if op == "orthogonalize":  # any matrix of a model, tall or wide
        D = round(_log_uniform(rng, 64, 8192))
        H = min(28672, max(64, round(D * _log_uniform(rng, 0.25, 4.0))))
        if rng.random() < 0.5:
            D, H = (D + 7) // 8 * 8, (H + 7) // 8 * 8
        return orthogonal(dtype, H, D)
    if op == "muon":
        D = max(256, round(_log_uniform(rng, 256, 8192) / 8) * 8)
        H = min(28672, round(D * rng.uniform(2.0, 4.0)))
        return muon(dtype, rng.randint(1, 16), H, D, master=dtype == "bf16" and rng.random() < 0.5, clip=rng.random() < 0.5,
                    nesterov=rng.random() < 0.75, scale=rng.choice(["spectral", "rms"]))
    types = rng.choice([("f32", "bf16", "bf16"), ("bf16", "bf16", "bf16"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "bf16"), ("f32", "f32", "f32")])
    post, pre = rng.choice([(True, True), (True, True), (True, False), (False, True)])
    D = max(64, round(_log_uniform(rng, 64, 8192) / 8) * 8)
    return norms(op, round(_log_uniform(rng, 1, 8192)), D, *types, gate=rng.choice(["none", "channel", "token", "full"]), post=post, pre=pre)


def _price(c):
    w = work(c)
    return w["bytes"] / 6.5e12 + w["flops"] / (6e13 if c.get("dtype") == "f32" else 1.4e15)


def draw(rng):
    every = listed()
    most = {op: max(_price(c) for c in every if c["op"] == op) for op in ("orthogonalize", "muon", "forward", "backward")}
    while True:
        c = _draw_once(rng)
        if _price(c) <= most[c["op"]]:
            return c


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(shape, std, dtype, gen):
    return torch.randn(shape, generator=gen, device=DEV).mul_(std).to(dtype)


def _gradient(H, D, gen):
    """The gradient of a matrix over 1024 tokens, fp32: one neuron in five fired for none of them, and features differ in size."""
    tokens = 1024
    fired = torch.rand(H, generator=gen, device=DEV) >= 0.2
    dz = torch.randn((tokens, H), generator=gen, device=DEV).mul_(fired)
    size = torch.randn(D, generator=gen, device=DEV).mul_(0.5).exp_()
    x = torch.randn((tokens, D), generator=gen, device=DEV).mul_(size)
    return (dz.T @ x).mul_(1e-4 / tokens)


def _prepare_muon(c, seed):
    gen, dtype = _gen(seed), DTYPES[c["dtype"]]
    n, H, D = 3 * c["layers"], c["H"], c["D"]
    whole = lambda t: torch.empty((n, H, D), dtype=t, device=DEV)  # noqa: E731  (the matrices are slices of one buffer)
    st = dict(op="muon", nesterov=c["nesterov"], scale=c["scale"], whole=dict(p=whole(dtype), m=whole(torch.float32)), grads=[])
    if c["master"]:
        st["whole"]["master"] = whole(torch.float32)
    st["params"], st["states"] = list(st["whole"]["p"]), [dict(m=m) for m in st["whole"]["m"]]
    st["masters"] = list(st["whole"]["master"]) if c["master"] else [None] * n
    for p, w, state in zip(st["params"], st["masters"], st["states"]):
        start = _normal((H, D), D ** -0.5, torch.float32, gen)
        p.copy_(start)
        if w is not None:
            w.copy_(start)
        st["grads"].append(_gradient(H, D, gen).to(dtype))
        # what earlier batches have left, most of it noise
        state["m"].copy_(_gradient(H, D, gen).mul_(0.3).add_(_normal((H, D), 1e-6, torch.float32, gen)))
    st["max_norm"] = MAX_NORM if c["clip"] else None
    st["grad_norm"] = 1.0 + torch.rand((), generator=gen, device=DEV) if c["clip"] else None
    return st


def _prepare_norms(c, seed):
    gen = _gen(seed)
    T, D, back = c["T"], c["D"], c["op"] == "backward"
    ty, ts, tn = (DTYPES[c[k]] for k in ("y", "stream", "out"))
    st = dict(op=c["op"], y=_normal((T, D), 0.3, ty, gen), n_dtype=tn)
    st["post_gain"] = 1.0 + 0.2 * torch.randn(D, generator=gen, device=DEV) if c["post"] else None
    st["pre_gain"] = 1.0 + 0.2 * torch.randn(D, generator=gen, device=DEV) if c["pre"] else None
    shape = {"none": None, "channel": (D,), "token": (T, 1), "full": (T, D)}[c["gate"]]
    st["gate"] = None if shape is None else (0.5 + 0.3 * torch.randn(shape, generator=gen, device=DEV)).to(ts if c["gate"] == "full" else torch.float32)
    size = torch.randn(D, generator=gen, device=DEV).mul_(0.5).exp_()  # channels of a residual stream differ in size
    h = torch.randn((T, D), generator=gen, device=DEV).mul_(size).mul_(2.0).to(ts)
    if not back:
        st["resid"] = h
        return st
    st["h"] = h  # what the forward pass saved, and what the two paths behind it hand back
    rstd = lambda v: (v.double().square().mean(1) + NORM_EPS).rsqrt().float()  # noqa: E731
    st["stats"] = torch.stack([rstd(st["y"]), rstd(h)])
    st["dh"] = _normal((T, D), 1.0 / T, ts, gen)
    st["dn"] = _normal((T, D), 1.0 / T, tn, gen) if c["pre"] else None
    return st


def prepare(c, seed):
    if c["op"] == "orthogonalize":
        return dict(op=c["op"], update=_gradient(c["H"], c["D"], _gen(seed)).to(DTYPES[c["dtype"]]))
    return _prepare_muon(c, seed) if c["op"] == "muon" else _prepare_norms(c, seed)


# ---- plain forms ---------------------------------------------------------------------------------------------------


def _orthogonal(u):
    """X = U / (|U| + eps), then X = a X + (b (X X^T) + c (X X^T)^2) X five times, on the shorter side."""
    a, b, c = COEFFICIENTS
    x = u.T if u.shape[0] > u.shape[1] else u
    x = x * (1.0 / (x.double().square().sum().sqrt() + EPS)).float()
    for _ in range(STEPS):
        p = x @ x.T
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.T if u.shape[0] > u.shape[1] else x


def _step_size(scale, shape):
    H, D = shape
    return math.sqrt(max(1.0, H / D)) if scale == "spectral" else 0.2 * math.sqrt(max(H, D))


def _muon(st):
    clip = None
    if st["max_norm"] is not None:
        clip = (st["max_norm"] / (st["grad_norm"] + 1e-6)).clamp(max=1.0)
    lr = LR[st["scale"]]
    for p, g, state, master in zip(st["params"], st["grads"], st["states"], st["masters"]):
        g = g.float()
        if clip is not None:
            g = g * clip
        m = state["m"] * MOMENTUM + g * (1.0 - MOMENTUM)
        u = m * MOMENTUM + g * (1.0 - MOMENTUM) if st["nesterov"] else m
        w = (p if master is None else master).float()
        w = w * (1.0 - lr * DECAY) - _orthogonal(u) * (lr * _step_size(st["scale"], p.shape))
        p.copy_(w)
        if master is not None:
            master.copy_(w)
        state["m"].copy_(m)
    return st["whole"]


def _rstd(v):
    return torch.rsqrt((v * v).mean(1) + NORM_EPS)


def _forward(st):
    y, resid = st["y"].float(), st["resid"].float()
    r = _rstd(y)
    v = y if st["post_gain"] is None else y * r[:, None] * st["post_gain"]
    if st["gate"] is not None:
        v = v * st["gate"].float()
    h = resid + v * KEEP
    out = dict(h=h.to(st["resid"].dtype))
    if st["pre_gain"] is not None:
        out["n"] = (h * _rstd(h)[:, None] * st["pre_gain"]).to(st["n_dtype"])
    return out


def _backward(st):
    y, h, g = st["y"].float(), st["h"].float(), st["dh"].float()
    D, out = y.shape[1], {}
    if st["pre_gain"] is not None:
        dn, r = st["dn"].float(), st["stats"][1][:, None]
        t = dn * st["pre_gain"]
        g = g + r * t - h * (r * r * r * ((t * h).sum(1, keepdim=True) / D))
        out["dpre_gain"] = (dn * h * r).sum(0)
    out["dresid"] = g.to(st["h"].dtype)
    normed = y if st["post_gain"] is None else y * st["stats"][0][:, None]
    v = normed if st["post_gain"] is None else normed * st["post_gain"]
    dv = g * KEEP
    if st["gate"] is not None:
        full, shape = dv * v, st["gate"].shape
        dgate = full if shape == full.shape else full.sum(0) if len(shape) == 1 else full.sum(1, keepdim=True)
        out["dgate"] = dgate.to(st["gate"].dtype)
        dv = dv * st["gate"].float()
    if st["post_gain"] is not None:
        out["dpost_gain"] = (dv * normed).sum(0)
        t, r = dv * st["post_gain"], st["stats"][0][:, None]
        dv = r * t - y * (r * r * r * ((t * y).sum(1, keepdim=True) / D))
    out["dy"] = dv.to(st["y"].dtype)
    return out


def run(st):
    if own:
        return _run_own(st)
    if st["op"] == "orthogonalize":
        return _orthogonal(st["update"].float()).to(st["update"].dtype)
    return {"muon": _muon, "forward": _forward, "backward": _backward}[st["op"]](st)


def _run_own(st):
    import paper_2609_31975_b200 as lib

    if st["op"] == "orthogonalize":
        return lib.orthogonalize(st["update"], steps=STEPS, coefficients=COEFFICIENTS, eps=EPS)
    if st["op"] == "muon":
        lib.muon_step(st["params"], st["grads"], st["states"], lr=LR[st["scale"]], momentum=MOMENTUM, nesterov=st["nesterov"], weight_decay=DECAY, scale=st["scale"],
                      steps=STEPS, coefficients=COEFFICIENTS, eps=EPS, masters=st["masters"], grad_norm=st["grad_norm"], max_norm=st["max_norm"])
        return st["whole"]
    if st["op"] == "forward":
        h, n, _ = lib.block_norm_forward(st["y"], st["resid"], st["post_gain"], st["pre_gain"], st["gate"], scale=KEEP, eps=NORM_EPS, n_dtype=st["n_dtype"])
        return dict(h=h) if n is None else dict(h=h, n=n)
    return lib.block_norm_backward(st["dh"], st["dn"], st["y"], st["h"], st["stats"], st["post_gain"], st["pre_gain"], st["gate"], scale=KEEP)


# ---- what a pass cannot do without ---------------------------------------------------------------------------------


def _products(rows, cols):
    """Operations of five Newton-Schulz steps of a matrix whose shorter side is s.  A step by itself: the Gram matrix and its square, of
    which half is enough, and the product with X.  Two at once: one Gram matrix, five such products of s x s, one product with X."""
    s, l = float(min(rows, cols)), float(max(rows, cols))
    one, two = 3 * l * s * s + s ** 3, 3 * l * s * s + 5 * s ** 3
    return STEPS // 2 * min(two, 2 * one) + STEPS % 2 * one


def work(c):
    if c["op"] == "orthogonalize":
        return {"bytes": 2.0 * c["H"] * c["D"] * ESZ[c["dtype"]], "flops": _products(c["H"], c["D"])}
    if c["op"] == "muon":
        # p read and written (with a copy in 32 bits that one is read and both are written), g read, m read and written
        e, n = ESZ[c["dtype"]], 3.0 * c["layers"] * c["H"] * c["D"]
        return {"bytes": n * ((10 if c["master"] else 2 * e) + e + 8), "flops": 3 * c["layers"] * _products(c["H"], c["D"])}
    n, (ey, es, en) = float(c["T"] * c["D"]), (ESZ[c[k]] for k in ("y", "stream", "out"))
    gate = es if c["gate"] == "full" else 0
    gains = 4.0 * c["D"] * (c["post"] + c["pre"] + (c["gate"] == "channel")) + 4.0 * c["T"] * (c["gate"] == "token")
    if c["op"] == "forward":  # y, resid, gate in; h, n out
        return {"bytes": n * (ey + 2 * es + gate + en * c["pre"]) + gains, "flops": 12 * n}
    # dh, dn, y, h, statistics, gate in; dresid, dy and the gradients of gains and gate out
    h = es if c["pre"] else 0
    return {"bytes": n * (2 * ey + 2 * es + h + en * c["pre"] + 2 * gate) + 2 * gains + 8.0 * c["T"], "flops": 24 * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------------------------


def _polar64(u):
    a, b, c = COEFFICIENTS
    rows, cols = u.shape
    x = u.double()
    x = x / (torch.linalg.vector_norm(x) + EPS)
    for _ in range(STEPS):
        if rows > cols:
            gram = torch.einsum("ki,kj->ij", x, x)
            poly = torch.einsum("ik,kj->ij", gram, gram).mul_(c).add_(gram, alpha=b)
            poly.diagonal().add_(a)
            x = torch.einsum("ik,kj->ij", x, poly)
        else:
            gram = torch.einsum("ik,jk->ij", x, x)
            poly = torch.einsum("ik,kj->ij", gram, gram).mul_(c).add_(gram, alpha=b)
            poly.diagonal().add_(a)
            x = torch.einsum("ik,kj->ij", poly, x)
    return x


def _exact_muon(c, seed):
    st = _prepare_muon(c, seed)
    clip = min(1.0, MAX_NORM / (float(st["grad_norm"]) + 1e-6)) if c["clip"] else 1.0
    n, H, D = 3 * c["layers"], c["H"], c["D"]
    out = {key: torch.empty((n, H, D), dtype=torch.float64, device=DEV) for key in ("p", "m")}
    lr, size = LR[c["scale"]], 0.2 * max(H, D) ** 0.5 if c["scale"] == "rms" else max(1.0, H / D) ** 0.5
    for i, (p, g, state, w) in enumerate(zip(st["params"], st["grads"], st["states"], st["masters"])):
        g = g.double() * clip
        m = out["m"][i].copy_(torch.lerp(g, state["m"].double(), MOMENTUM))
        o = _polar64(torch.lerp(g, m, MOMENTUM) if c["nesterov"] else m)
        out["p"][i].copy_((p if w is None else w).double() * (1 - lr * DECAY) - o.mul_(lr * size))
    if c["master"]:
        out["master"] = out["p"]
    return out


def _exact_norms(c, seed):
    st = _prepare_norms(c, seed)
    wide = lambda k: None if st[k] is None else st[k].double()  # noqa: E731
    y, post, pre, gate = wide("y"), wide("post_gain"), wide("pre_gain"), wide("gate")
    T, D = y.shape
    factor = KEEP * (torch.ones((1, 1), dtype=torch.float64, device=DEV) if gate is None else gate.expand(T, D) if gate.dim() == 2 else gate[None])
    if c["op"] == "forward":
        z = y if post is None else y / (torch.linalg.vector_norm(y, dim=1, keepdim=True) ** 2 / D + NORM_EPS) ** 0.5 * post
        h = wide("resid") + factor * z
        if pre is None:
            return dict(h=h)
        return dict(h=h, n=h / (torch.linalg.vector_norm(h, dim=1, keepdim=True) ** 2 / D + NORM_EPS) ** 0.5 * pre)
    h, total, out = wide("h"), wide("dh"), {}
    ry, rh = st["stats"].double()
    if pre is not None:
        unit, back = h * rh[:, None], wide("dn") * pre
        out["dpre_gain"] = torch.einsum("td,td->d", wide("dn"), unit)
        total = total + rh[:, None] * (back - unit * torch.einsum("td,td->t", back, unit)[:, None] / D)
    out["dresid"] = total
    unit = y if post is None else y * ry[:, None]
    z = unit if post is None else unit * post
    if gate is not None:
        out["dgate"] = KEEP * (total * z if gate.shape == z.shape and gate.dim() == 2 and c["gate"] == "full" else torch.einsum("td,td->d", total, z)
                               if gate.dim() == 1 else torch.einsum("td,td->t", total, z)[:, None])
    dz = total * factor
    if post is not None:
        out["dpost_gain"] = torch.einsum("td,td->d", dz, unit)
        back = dz * post
        dz = ry[:, None] * (back - unit * torch.einsum("td,td->t", back, unit)[:, None] / D)
    out["dy"] = dz
    return out


def exact(c, seed):
    if c["op"] == "orthogonalize":
        return _polar64(prepare(c, seed)["update"])
    return _exact_muon(c, seed) if c["op"] == "muon" else _exact_norms(c, seed)
