"""GPU parity of the orthogonalised update and the Muon step with their formulas in 64 bits.  Run with `-m gpu` on a B200."""
import math

import pytest
import torch

import muon_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
SHORT = 2_000_000        # cycles: about a millisecond


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    yield m
    assert m.training_status(DEV) == 0


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def normal(shape, g, std=1.0, dtype=F32):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


SHAPES = [(1, 1), (1, 8), (8, 1), (3, 5), (16, 16), (33, 70), (70, 33), (64, 300), (129, 128), (256, 256), (257, 300), (300, 257), (1024, 256), (256, 1024),
          (513, 520), (1000, 640), (640, 1000), (767, 2050), (2050, 767), (1300, 1290), (4096, 700), (700, 4096)]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
def test_shapes(lib, shape, dtype):
    u = normal(shape, gen(shape[0] + shape[1]), 1e-3, dtype)
    got = lib.orthogonalize(u)
    assert got.dtype == dtype
    ref.close(got, ref.orthogonal(u), 32 if dtype == F32 else 16)


def spectra(R, C, g):
    S = min(R, C)
    q, _ = torch.linalg.qr(torch.randn((R, S), generator=g, device=DEV, dtype=torch.float64))
    p, _ = torch.linalg.qr(torch.randn((C, S), generator=g, device=DEV, dtype=torch.float64))
    i = torch.arange(1, S + 1, device=DEV, dtype=torch.float64)
    for name, s in (("one", torch.ones_like(i)), ("root", i ** -0.5), ("inverse", 1 / i), ("square", i ** -2), ("rank 1", (i == 1).double()), ("rank 7", (i <= 7).double()),
                    ("two sizes", torch.where(i < S / 2, 1.0, 1e-3))):
        yield name, (q * s) @ p.T
    dead = torch.randn((R, C), generator=g, device=DEV, dtype=torch.float64)
    dead[::2] = 0
    dead[:, 5:9] = 0
    yield "dead", dead
    yield "heavy", torch.randn((R, C), generator=g, device=DEV, dtype=torch.float64) * torch.exp(2 * torch.randn((R, 1), generator=g, device=DEV, dtype=torch.float64))


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("shape", [(600, 300), (300, 600), (520, 520)], ids=str)
def test_spectra(lib, shape, bits):
    """Singular values far apart, few of them, rows and columns of zeros: what lies far below the largest is not lost in its roundings."""
    for name, u in spectra(*shape, gen(3)):
        for dtype in (F32, BF16):
            v = u.to(dtype)
            try:
                ref.close(lib.orthogonalize(v, bits=bits), ref.orthogonal(v), bits)
            except AssertionError as e:
                raise AssertionError(f"{name}, {dtype}: {e}") from e


@pytest.mark.parametrize("size", [1e-42, 1e-30, 1e-12, 1.0, 1e15, 1e34])
def test_sizes_of_values(lib, size):
    """The update's size does not matter: eps is zero here, as next to 1e-30 it would be all there is."""
    u = (torch.randn((200, 96), generator=gen(1), device=DEV, dtype=torch.float64) * size).float()
    ref.close(lib.orthogonalize(u, eps=0.0), ref.orthogonal(u, eps=0.0), 32)
    small = lib.orthogonalize(u, eps=1e-7)
    ref.close(small, ref.orthogonal(u, eps=1e-7), 32, a=3.4445)


def test_zeros_and_what_is_not_finite(lib):
    for dtype in (F32, BF16):
        z = torch.zeros((300, 40), device=DEV, dtype=dtype)
        assert not lib.orthogonalize(z).any() and not lib.orthogonalize(z, eps=0.0).any()
        for bad in (float("nan"), float("inf")):
            u = normal((300, 40), gen(2), dtype=dtype)
            u[17, 3] = bad
            good = normal((300, 40), gen(4), dtype=dtype)
            a, b = lib.orthogonalize([u, good])
            assert a.isnan().all() and torch.equal(b, lib.orthogonalize([good, good])[1])
        for shape in ((0, 8), (8, 0), (0, 0)):
            assert lib.orthogonalize(torch.zeros(shape, device=DEV, dtype=dtype)).shape == shape
    assert lib.orthogonalize([]) == []


@pytest.mark.parametrize("steps,coefficients", [(1, ref.COEFFICIENTS), (2, (1.5, -0.5, 0.0)), (8, (1.5, -0.5, 0.0)), (3, (0.0, 0.0, 0.0)), (4, (2.0, -1.5, 0.5)), (1, (1.0, 0.0, 0.0)),
                                                (3, [(4.0, -6.0, 3.0), (3.5, -5.0, 2.2), (1.875, -1.25, 0.375)]), (2, (30.0, 2.0, 5.0))])
def test_coefficients(lib, steps, coefficients):
    most = max(c[0] for c in coefficients) if hasattr(coefficients[0], "__len__") else coefficients[0]
    for shape in ((90, 200), (320, 144)):
        u = normal(shape, gen(steps))
        want = ref.orthogonal(u, steps, coefficients)
        for bits in (16, 32):
            got = lib.orthogonalize(u, steps=steps, coefficients=coefficients, bits=bits)
            if want.any():
                ref.close(got, want, bits, steps, most)
            else:
                assert not got.any()


def test_lists_of_every_kind(lib):
    """Shapes and types mixed, more of one shape than a launch takes: each as by itself up to the order of sums, and in its place."""
    g = gen(8)
    us = [normal((40, 24), g, dtype=BF16 if i % 7 == 3 else F32) for i in range(150)]
    us += [normal((24, 40), g), torch.zeros((0, 24), device=DEV), normal((200, 330), g, dtype=BF16), normal((1, 1), g)]
    order = torch.randperm(len(us), generator=torch.Generator().manual_seed(1)).tolist()
    us = [us[i] for i in order]
    got, again = lib.orthogonalize(us), lib.orthogonalize(us)
    for u, o, o2 in zip(us, got, again):
        assert torch.equal(o, o2) and o.dtype == u.dtype
        ref.close(o, ref.orthogonal(u) if u.numel() else u.double(), 32 if u.dtype == F32 else 16)


def test_rows_apart_and_in_place(lib):
    """Strided rows at any alignment, columns of one matrix as outputs, an update that is its own output; nothing else is written."""
    g = gen(5)
    for dtype in (F32, BF16):
        for shape in ((150, 70), (70, 150)):
            R, C = shape
            u = normal(shape, g, dtype=dtype)
            want = lib.orthogonalize(u)
            room = torch.full((R + 2, 2 * C + 9), 7.0, device=DEV, dtype=dtype)
            a, b = room[1:-1, 1:C + 1], room[1:-1, C + 3:2 * C + 3]
            a.copy_(u)
            keep = room.clone()
            x, y = lib.orthogonalize([a, u], out=[a, b])
            assert x is a or x.data_ptr() == a.data_ptr()
            keep[1:-1, 1:C + 1], keep[1:-1, C + 3:2 * C + 3] = a, b
            assert torch.equal(room, keep)
            two = lib.orthogonalize([u, u])
            assert torch.equal(a, two[0]) and torch.equal(b, two[1])
            ref.close(a, ref.orthogonal(u), 32 if dtype == F32 else 16)
            got = lib.orthogonalize(u, out=u)
            assert got.data_ptr() == u.data_ptr() and torch.equal(u, want)


STEP = dict(lr=0.02, momentum=0.9, nesterov=True, weight_decay=0.1)


def tensors(shape, kind, g):
    """kind: f32, bf16, master (bf16 with a copy)."""
    start = normal(shape, g, shape[1] ** -0.5)
    p = start.clone() if kind == "f32" else start.bfloat16()
    return p, normal(shape, g, 1e-3, F32 if kind == "f32" else BF16), dict(m=normal(shape, g, 3e-4)), start.clone() if kind == "master" else None


def check_step(before, after, how, scale, bits, clip=1.0, ns=None):
    p, g, state, w = before
    want, m = ref.step(p, g, state["m"], w, scale=scale, clip=clip, **how, **(ns or {}))
    o = (p if w is None else w).double() * (1 - how["lr"] * how["weight_decay"]) - want      # what the step takes away
    limit = ref.room(bits, 5, ref.COEFFICIENTS[0], (o.norm() / (how["lr"] * scale)).item()) * o.norm().item()
    q, _, after_state, after_w = after
    # moments: three roundings of their terms; the parameter: four, and its own
    assert (after_state["m"].double() - m).abs().max() <= 4 * 2.0 ** -24 * (m.abs() + state["m"].abs() + g.double().abs() * clip).max()
    for t in [q] + ([after_w] if w is not None else []):
        own = torch.finfo(t.dtype).eps / 2
        assert (t.double() - want).norm() <= limit + (own + 4 * 2.0 ** -24) * (want.abs() + o.abs()).norm(), (t.dtype,)
    if w is not None:
        assert torch.equal(q, after_w.bfloat16())


def copy(t):
    p, g, state, w = t
    return p.clone(), g.clone(), dict(m=state["m"].clone()), None if w is None else w.clone()


@pytest.mark.parametrize("kind", ["f32", "bf16", "master"])
@pytest.mark.parametrize("bits", [None, 16, 32])
def test_steps(lib, kind, bits):
    for shape in ((300, 120), (120, 300), (65, 33)):
        for how in (STEP, dict(STEP, nesterov=False), dict(STEP, momentum=0.0, weight_decay=0.0)):
            t = tensors(shape, kind, gen(shape[0]))
            before = copy(t)
            lib.muon_step([t[0]], [t[1]], [t[2]], masters=None if t[3] is None else [t[3]], scale=1.5, bits=bits, **how)
            check_step(before, t, how, 1.5, bits or (16 if kind == "bf16" else 32))
            assert torch.equal(before[1], t[1])


def test_a_list_with_rules_and_clipping(lib):
    """A model's matrices, bf16 with and without copies, fp32: learning rates of their own, a rule for the size, gradients scaled by their
    norm.  A norm that is not finite leaves everything as it was."""
    g = gen(11)
    kinds = ["master", "bf16", "f32", "master", "bf16", "f32", "bf16"]
    shapes = [(256, 64), (256, 64), (256, 64), (256, 64), (64, 200), (31, 77), (256, 64)]
    ts = [tensors(s, k, g) for s, k in zip(shapes, kinds)]
    rates = [0.02 + 0.01 * i for i in range(len(ts))]
    norm = lib.grad_norm([t[1] for t in ts])
    clip = 0.01 / (norm.item() + 1e-6)
    assert clip < 1
    columns = [list(c) for c in zip(*ts)]

    def step(norm, scale):
        lib.muon_step(columns[0], columns[1], columns[2], lr=rates, momentum=0.9, weight_decay=0.1, scale=scale, masters=columns[3], grad_norm=norm, max_norm=0.01)

    before = [copy(t) for t in ts]
    step(norm, "rms")
    for a, b, s, k, r in zip(before, ts, shapes, kinds, rates):
        check_step(a, b, dict(STEP, lr=r), 0.2 * math.sqrt(max(s)), 16 if k == "bf16" else 32, clip)
    before = [copy(t) for t in ts]
    for bad in (float("nan"), float("inf")):
        step(torch.tensor(bad, device=DEV), "spectral")
    for a, b in zip(before, ts):
        assert torch.equal(a[0], b[0]) and torch.equal(a[2]["m"], b[2]["m"]) and (a[3] is None or torch.equal(a[3], b[3]))
    step(norm, "spectral")
    for a, b, s, k, r in zip(before, ts, shapes, kinds, rates):
        check_step(a, b, dict(STEP, lr=r), math.sqrt(max(1.0, s[0] / s[1])), 16 if k == "bf16" else 32, clip)


def test_slices_that_start_anywhere(lib):
    """Parameters at any alignment of their type, neighbours in one buffer."""
    for kind in ("f32", "bf16", "master"):
        shape, n = (45, 30), 45 * 30
        want = tensors(shape, kind, gen(6))
        room = {k: torch.full((n + 20,), 7.0, device=DEV, dtype=v.dtype) for k, v in (("p", want[0]), ("g", want[1]), ("m", want[2]["m"]), ("w", want[2]["m"]))}
        at = dict(p=3, g=5, m=1, w=7)
        s = {k: room[k][at[k]:at[k] + n].view(shape) for k in room}
        for k, v in (("p", want[0]), ("g", want[1]), ("m", want[2]["m"]), ("w", want[3])):
            if v is not None:
                s[k].copy_(v)
        lib.muon_step([want[0]], [want[1]], [want[2]], masters=[want[3]], **STEP)
        lib.muon_step([s["p"]], [s["g"]], [dict(m=s["m"])], masters=[s["w"] if want[3] is not None else None], **STEP)
        assert torch.equal(s["p"], want[0]) and torch.equal(s["m"], want[2]["m"]) and (want[3] is None or torch.equal(s["w"], want[3]))
        for k, r in room.items():
            assert (r[:at[k]] == 7).all() and (r[at[k] + n:] == 7).all(), k


def test_other_streams_and_a_graph(lib):
    t = tensors((300, 200), "master", gen(1))
    u = t[1].clone()
    start = copy(t)
    lib.muon_step([t[0]], [t[1]], [t[2]], masters=[t[3]], **STEP)
    want, o = copy(t), lib.orthogonalize(u)

    def restart():
        for a, b in ((t[0], start[0]), (t[2]["m"], start[2]["m"]), (t[3], start[3])):
            a.copy_(b)

    def same():
        return torch.equal(t[0], want[0]) and torch.equal(t[2]["m"], want[2]["m"]) and torch.equal(t[3], want[3])

    side = torch.cuda.Stream()
    restart()
    torch.cuda.synchronize()
    lib.muon_step([t[0]], [t[1]], [t[2]], masters=[t[3]], stream=side, **STEP)
    o2 = lib.orthogonalize(u, stream=side)
    side.synchronize()
    assert same() and torch.equal(o, o2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lib.muon_step([t[0]], [t[1]], [t[2]], masters=[t[3]], **STEP)
        o3 = lib.orthogonalize(u)
    for _ in range(2):
        restart()
        graph.replay()
        torch.cuda.synchronize()
        assert same() and torch.equal(o, o3)


def test_torch_sees_what_is_written(lib):
    t = tensors((64, 32), "f32", gen(1))
    leaf = t[0].requires_grad_()
    y = (leaf * leaf).sum()
    with torch.no_grad():
        lib.muon_step([leaf], [t[1]], [t[2]], **STEP)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def test_a_copy_that_never_comes(lib):
    """A wait that runs out ends the call with a status, gives tensor memory back, and the next call computes as before."""
    try:
        for dtype in (BF16, F32):
            u = normal((700, 520), gen(1), dtype=dtype)
            want = lib.orthogonalize(u)
            assert lib.training_status(DEV) == 0
            lib.test_set_knob("wait_cycles", SHORT)
            lib.test_set_knob("drop_stage", 0)  # (the small products here are cut into pieces of one K block: a CTA has no other)
            lib.orthogonalize(u)
            assert lib.training_status(DEV, reset=True) == 5
            lib.test_set_knob("wait_cycles", 0)
            lib.test_set_knob("drop_stage", -1)
            assert torch.equal(lib.orthogonalize(u), want) and lib.training_status(DEV) == 0
    finally:
        lib.test_set_knob("wait_cycles", 0)
        lib.test_set_knob("drop_stage", -1)
        lib.training_status(DEV, reset=True)


def test_refusals(lib):
    u = normal((64, 32), gen(1))
    for bad in (u.half(), u.cpu(), u[0], u[None], u.t().contiguous().t()):
        with pytest.raises(TypeError):
            lib.orthogonalize(bad)
    for how in (dict(steps=0), dict(coefficients=[(1, 2, 3)] * 4), dict(coefficients=(1, 2))):
        with pytest.raises(ValueError):
            lib.orthogonalize(u, **how)
    for how in (dict(steps=33), dict(eps=-1.0), dict(eps=float("nan")), dict(bits=8), dict(coefficients=(50.0, 50.0, 50.0)), dict(coefficients=(1.0, float("nan"), 0.0))):
        with pytest.raises(lib.SFFNError):
            lib.orthogonalize(u, **how)
    o = torch.empty_like(u)
    for us, outs in (([u, u], [o, o]), ([u, o], [u.clone(), u]), ([u], [u[1:2].expand(64, 32)])):
        with pytest.raises((lib.SFFNError, TypeError)):
            lib.orthogonalize(us, outs)
    with pytest.raises(ValueError):
        lib.orthogonalize([u], [])
    with pytest.raises(TypeError):
        lib.orthogonalize(u, out=o.bfloat16())
    t = tensors((64, 32), "master", gen(1))
    before = copy(t)
    ok = ([t[0]], [t[1]], [t[2]])
    for args, how in ((([t[0][0]], [t[1][0]], [dict(m=t[2]["m"][0])]), {}), (([t[0]], [t[1][:5]], [t[2]]), {}), (([t[0]], [t[1]], [dict(m=t[2]["m"].bfloat16())]), {}),
                      (([t[0]], [t[1]], [{}]), {}), (([t[0]], [t[1]], [t[2]["m"]]), {}), (ok, dict(masters=[t[3].bfloat16()])), (([t[0].cpu()], [t[1]], [t[2]]), {}),
                      (([t[0].t()], [t[1].t()], [dict(m=t[2]["m"].t())]), {})):
        with pytest.raises(TypeError):
            lib.muon_step(*args, **{**STEP, **how})
    for args, how in (((ok[0], [], ok[2]), {}), (ok, dict(lr=[0.1, 0.2])), (ok, dict(scale="other")), (ok, dict(scale=[1.0, 2.0])), (ok, dict(max_norm=1.0)), (([], [t[1]], []), {})):
        with pytest.raises(ValueError):
            lib.muon_step(*args, **{**STEP, **how})
    for args, how in ((ok, dict(momentum=1.0)), (ok, dict(lr=float("nan"))), (ok, dict(grad_norm=torch.ones((), device=DEV), max_norm=0.0)), (ok, dict(steps=40)),
                      (([t[0], t[0]], [t[1], t[1]], [t[2], dict(m=t[2]["m"].clone())]), {}), (([t[0]], [t[0]], [t[2]]), {}),
                      (([t[0]], [t[1]], [t[2]]), dict(masters=[t[2]["m"]])), (([t[3]], [t[1]], [t[2]]), dict(masters=[t[2]["m"].clone()]))):
        with pytest.raises(lib.SFFNError):
            lib.muon_step(*args, **{**STEP, **how})
    assert torch.equal(t[0], before[0]) and torch.equal(t[2]["m"], before[2]["m"]) and torch.equal(t[3], before[3])
    lib.muon_step([], [], [], lr=0.1)
