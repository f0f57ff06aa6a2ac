"""GPU parity of the gradient norm and the AdamW step with their formulas in 64 bits.  Run with `-m gpu` on a B200."""
import math

import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    return m


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def slices(n, dtype, offset, g, std=1.0):
    """n entries that start `offset` entries into their buffer."""
    t = (torch.randn(n + offset, generator=g, device=DEV) * std).to(dtype)
    return t[offset:]


SIZES = [1, 3, 255, 256, 257, 511, 2048, 100003]


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("offset", [0, 1, 4])
def test_norm_of_many_sizes(lib, dtype, offset):
    """Entries are squared and summed in fp32 over at most 64 * 32 terms, then in fp64: within 2048 units of 2^-24 in the sum, in
    truth a few; half of that in the root, and one rounding."""
    for n in SIZES + [1 << 20, 3000001]:
        t = slices(n, dtype, offset, gen(n + offset))
        got = lib.grad_norm([t]).item()
        want = t.double().norm().item()
        assert abs(got - want) <= 1024 * ref.U32 * want, (n, got, want)
        assert abs(got - want) <= 1e-6 * want, (n, got, want)


def test_norm_of_lists(lib):
    g = gen(1)
    for count in (1, 2, 39, 40, 41, 500, 1299, 1300, 1301, 2700):
        ts = [slices(1 + (37 * i) % 700, BF16 if i % 3 else F32, 0, g) for i in range(count)]
        ts.insert(count // 2, torch.empty(0, device=DEV))
        want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in ts))
        a, b = lib.grad_norm(ts), lib.grad_norm(ts)
        assert abs(a.item() - want) <= 1e-6 * want and torch.equal(a, b), count
    assert lib.grad_norm([torch.empty(0, device=DEV)]).item() == 0.0
    z = torch.zeros(1000, device=DEV)
    assert lib.grad_norm([z]).item() == 0.0
    z[777] = float("inf")
    assert lib.grad_norm([z]).item() == math.inf
    z[5] = float("nan")
    assert math.isnan(lib.grad_norm([z]).item())
    assert lib.grad_norm([torch.full((3,), 1e25, device=DEV)]).item() == math.inf      # squares leave fp32
    side = torch.cuda.Stream()
    t = slices(12345, F32, 0, g)
    torch.cuda.synchronize()
    assert lib.grad_norm([t], stream=side).item() == lib.grad_norm([t]).item()


def tensors(lib, n, p_dtype, g_dtype, bits, master, offset, seed, zero_groups=False):
    g = gen(seed)
    start = torch.randn(n + offset, generator=g, device=DEV)
    p = start.to(p_dtype)[offset:]
    w = start.clone()[offset:] if master else None
    grad = slices(n, g_dtype, offset, g, 1e-3)
    if zero_groups:
        grad[: n // 2] = 0
    if bits == 32:
        state = dict(m=slices(n, F32, offset, g, 1e-3), v=slices(n, F32, offset, g, 1e-3).square())
    else:
        groups = -(-n // 256)
        state = dict(m=torch.randint(-127, 128, (n + offset,), generator=g, device=DEV).to(torch.int8)[offset:],
                     v=torch.randint(0, 256, (n + offset,), generator=g, device=DEV).to(torch.uint8)[offset:],
                     m_scale=torch.rand(groups, generator=g, device=DEV) * 1e-3, v_scale=torch.rand(groups, generator=g, device=DEV) * 1e-6)
        if zero_groups:
            for k in ("m_scale", "v_scale"):
                state[k][: groups // 2] = 0
            state["m"][: groups // 2 * 256] = 0
            state["v"][: groups // 2 * 256] = 0
    return p, grad, state, w


def values(state):
    if "m_scale" in state:
        return ref.decode(state["m"], state["m_scale"], 127, 2), ref.decode(state["v"], state["v_scale"], 255, 4)
    return state["m"].cpu().double(), state["v"].cpu().double()


HYPER = dict(lr=1e-2, betas=(0.9, 0.98), eps=1e-8, weight_decay=0.1)


def copied(state):
    return {k: t.clone() for k, t in state.items()}


def check(before, after, step, scale, what, hyper=HYPER):
    """m and v carry four fp32 roundings of the terms they are made of; p those, and some units of a root and a quotient on the
    step's part.  8-bit moments come back within half a code, the fourth root of which is half of 1 / 255 of the scale's."""
    (p0, g, s0, w0), (p1, s1, w1) = before, after
    m0, v0 = values(s0)
    start = p0 if w0 is None else w0
    p, m, v = ref.adamw(start, g, m0, v0, step, hyper["lr"], hyper["betas"], hyper["eps"], hyper["weight_decay"], scale)
    b1, b2 = hyper["betas"]
    g64 = g.cpu().double() * scale
    terms = b1 * m0.abs() + (1 - b1) * g64.abs()
    em = 8 * ref.U32 * terms
    ev = 10 * ref.U32 * v
    root = (v / (1 - b2 ** step)).sqrt() + hyper["eps"]
    part = hyper["lr"] / (1 - b1 ** step) * (em + 32 * ref.U32 * m.abs()) / root
    ep = part + 4 * ref.U32 * (start.cpu().double().abs() + (p - start.cpu().double()).abs()) + 1e-44
    got = (p1 if w1 is None else w1).cpu().double()
    out = ref.U16 * (p.abs() + ep) if p1.dtype == BF16 and w1 is None else 0
    assert ((got - p).abs() <= ep + out).all(), (what, float(((got - p).abs() - ep - out).max()))
    if w1 is not None:
        assert torch.equal(p1, w1.to(BF16)), what
    m1, v1 = values(s1)
    if "m_scale" not in s1:
        assert ((m1 - m).abs() <= em + 1e-44).all() and ((v1 - v).abs() <= ev + 1e-44).all(), what
        return
    n = m.numel()
    for new, want, scale_, levels, power, e in ((m1, m, s1["m_scale"], 127, 2, em), (v1, v, s1["v_scale"], 255, 4, ev)):
        s = scale_.cpu().double()
        most = torch.stack([b.abs().max() for b in want.split(256)])
        assert ((s - most).abs() <= 1e-5 * most).all(), (what, levels)
        s = s.repeat_interleave(256)[:n]
        fine = s > 0
        assert (want[~fine].abs() < 2.0 ** -99).all()
        root_new = (new[fine].abs() / s[fine]) ** (1 / power) * levels
        root_want = (want[fine].abs() / s[fine]) ** (1 / power) * levels
        near = (root_new - root_want).abs() <= 0.5 + 1e-2
        if levels == 255:  # what is not zero keeps a code
            near |= (root_new - 1).abs() < 1e-3
            assert ((new[fine] > 0) == (want[fine] > 0)).all(), what
        assert near.all(), (what, levels, float((root_new - root_want).abs().max()))
        assert ((new[fine] * want[fine] >= 0)).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_dtype,g_dtype,master", [(F32, F32, False), (F32, BF16, False), (BF16, BF16, False), (BF16, F32, False), (BF16, BF16, True)],
                         ids=["f32", "f32_gbf16", "bf16", "bf16_gf32", "master"])
@pytest.mark.parametrize("offset", [0, 1, 8])
def test_one_step(lib, bits, p_dtype, g_dtype, master, offset):
    for n in SIZES:
        p, g, s, w = tensors(lib, n, p_dtype, g_dtype, bits, master, offset, n + offset, zero_groups=n % 2 == 0)
        before = (p.clone(), g.clone(), copied(s), None if w is None else w.clone())
        lib.adamw_step([p], [g], [s], 3, masters=[w], **HYPER)
        torch.cuda.synchronize()
        check(before, (p, s, w), 3, 1.0, (n, bits, offset))
        assert torch.equal(before[1], g)


def test_lists_groups_and_clipping(lib):
    for count in (2, 40, 41, 359, 361, 800):
        rows = [tensors(lib, 1 + (91 * i) % 1500, F32 if i % 4 == 0 else BF16, BF16 if i % 4 else F32, 8 if i % 2 else 32, i % 4 == 3, 0, i) for i in range(count)]
        before = [(p.clone(), g.clone(), copied(s), None if w is None else w.clone()) for p, g, s, w in rows]
        ps, gs, ss, ws = (list(c) for c in zip(*rows))
        norm = lib.grad_norm(gs)
        lrs, wds = [1e-3 * (1 + i % 3) for i in range(count)], [0.1 * (i % 2) for i in range(count)]
        most = norm.item() / 3
        lib.adamw_step(ps, gs, ss, 17, lr=lrs, betas=(0.9, 0.98), eps=1e-8, weight_decay=wds, masters=ws, grad_norm=norm, max_norm=most)
        torch.cuda.synchronize()
        for i in list(range(0, count, 7)) + [count - 1]:
            check(before[i], (ps[i], ss[i], ws[i]), 17, min(1.0, most / (norm.item() + 1e-6)), (count, i), dict(HYPER, lr=lrs[i], weight_decay=wds[i]))


@pytest.mark.parametrize("bits", [32, 8])
def test_a_norm_that_is_not_finite_leaves_everything(lib, bits):
    for bad in (math.inf, math.nan):
        p, g, s, w = tensors(lib, 5000, BF16, BF16, bits, True, 0, 4)
        keep = [p.clone(), w.clone(), copied(s)]
        g[4321] = bad
        lib.adamw_step([p], [g], [s], 1, masters=[w], grad_norm=lib.grad_norm([g]), max_norm=1.0, **HYPER)
        torch.cuda.synchronize()
        assert torch.equal(p, keep[0]) and torch.equal(w, keep[1]) and all(torch.equal(s[k], keep[2][k]) for k in s)
    p, g, s, w = tensors(lib, 5000, BF16, BF16, bits, True, 0, 4)
    g[4321] = math.nan       # without a norm it goes where it belongs, and no further than its group
    lib.adamw_step([p], [g], [s], 1, masters=[w], **HYPER)
    torch.cuda.synchronize()
    assert torch.isnan(w).nonzero().tolist() == [[4321]]
    m, v = values(s)
    group = slice(4321 // 256 * 256, 4321 // 256 * 256 + 256)
    outside = torch.ones(5000, dtype=torch.bool)
    outside[group] = False
    assert torch.isfinite(m[outside]).all() and torch.isfinite(v[outside]).all() and torch.isnan(m[4321]) and torch.isnan(v[4321])


def test_codes_are_the_nearest_ones_exactly(lib):
    """The codes against the edges (k + 1/2)^2 and (k + 1/2)^4 in fp32 arithmetic: equal, entry by entry."""
    n = 1 << 18
    p, g, s, _ = tensors(lib, n, F32, F32, 8, False, 0, 77)
    g[: 256 * 40] = (g[: 256 * 40].view(40, 256) * torch.logspace(0, -12, 40, device=DEV)[:, None]).reshape(-1)
    g[256 * 50: 256 * 60] *= torch.logspace(0, -8, 2560, device=DEV)
    m0 = (s["m"].float() * s["m"].float().abs()).view(-1, 256) * (s["m_scale"] * (1.0 / 127.0 ** 2))[:, None]
    v0 = (s["v"].float() * s["v"].float()).square().view(-1, 256) * (s["v_scale"] * (1.0 / 255.0 ** 4))[:, None]
    gg = g.view(-1, 256)
    m = m0 * 0.9 + gg * (1.0 - 0.9)
    v = v0 * 0.999 + gg * gg * (1.0 - 0.999)
    lib.adamw_step([p], [g], [s], 5, lr=1e-3)
    k = torch.arange(255, device=DEV, dtype=F32)
    edges = k * k + k + 0.25
    for t, top, e, codes, scale in ((m, 127.0 ** 2, edges[:127], s["m"], s["m_scale"]), (v, 255.0 ** 4, edges.square(), s["v"], s["v_scale"])):
        most = t.abs().amax(1)
        assert torch.equal(scale, most)
        q = t.abs() * most.reciprocal()[:, None] * top
        want = torch.bucketize(q, e, right=True)
        if codes.dtype == torch.uint8:
            want = torch.where(t > 0, want.clamp(min=1), want)
        else:
            want = want * t.sign().long()
        assert torch.equal(codes.view(-1, 256).long(), want)


def test_values_of_8_bit_moments(lib):
    for count, offset in ((1, 0), (1, 1), (45, 0), (400, 0)):
        states = [tensors(lib, 1 + (433 * i + 1000 * (count == 1)) % 3000, F32, F32, 8, False, offset, i)[2] for i in range(count)]
        got = lib.adamw_state_values(states)
        torch.cuda.synchronize()
        for s, o in zip(states, got):
            m, v = values(s)
            assert ((o["m"].cpu().double() - m).abs() <= 4 * ref.U32 * m.abs()).all() and ((o["v"].cpu().double() - v).abs() <= 4 * ref.U32 * v.abs()).all()


def test_training_runs_down_with_moments_in_8_bits(lib):
    """A least-squares problem over a rotated basis: 8-bit moments come as low as moments in 32 bits do, within a factor."""
    g = gen(9)
    A = torch.randn(512, 256, generator=g, device=DEV) / 16
    target = A @ torch.randn(256, 64, generator=g, device=DEV)
    final = {}
    for bits in (32, 8):
        w = torch.zeros(256, 64, device=DEV)
        s = lib.adamw_state(w, bits)
        for k in range(1, 301):
            grad = A.T @ (A @ w - target)
            lib.adamw_step([w], [grad], [s], k, lr=2e-2, weight_decay=0.0)
        final[bits] = ((A @ w - target) ** 2).mean().item() / (target ** 2).mean().item()
    assert final[32] < 1e-2 and final[8] < 3 * final[32] + 1e-3, final


def test_in_a_graph(lib):
    p, g, s, _ = tensors(lib, 70000, F32, F32, 8, False, 0, 3)
    q, h, r, _ = tensors(lib, 70000, F32, F32, 8, False, 0, 3)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = lib.grad_norm([g])
        lib.adamw_step([p], [g], [s], 2, grad_norm=norm, max_norm=0.1, **HYPER)
    for _ in range(3):
        graph.replay()
        lib.adamw_step([q], [h], [r], 2, grad_norm=lib.grad_norm([h]), max_norm=0.1, **HYPER)
    torch.cuda.synchronize()
    assert torch.equal(p, q) and all(torch.equal(s[k], r[k]) for k in s)


def test_refusals(lib):
    p, g, s, w = tensors(lib, 512, BF16, BF16, 32, True, 0, 1)
    step = lambda *a, **k: lib.adamw_step(*a, **dict(HYPER, **k))  # noqa: E731
    with pytest.raises(TypeError):
        step([p], [g.half()], [s], 1)
    with pytest.raises(TypeError):
        step([p], [g[:500]], [s], 1)
    with pytest.raises(TypeError):
        step([p], [g], [dict(s, m=s["m"].half())], 1)
    with pytest.raises(ValueError):
        step([p, p], [g], [s], 1)
    with pytest.raises(ValueError):
        step([p], [g], [s], 1, max_norm=1.0)
    for bad in (dict(step=0), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(lr=math.nan)):
        with pytest.raises(lib.SFFNError) as err:
            step([p], [g], [s], bad.pop("step", 1), **bad)
        assert err.value.code == 1
    with pytest.raises(lib.SFFNError):                                   # a master copy of what is fp32 itself
        step([w], [g], [s], 1, masters=[w.clone()])
    with pytest.raises(lib.SFFNError):
        step([p], [g], [s], 1, grad_norm=lib.grad_norm([g]), max_norm=0.0)
    with pytest.raises(ValueError):
        lib.grad_norm([])
    with pytest.raises(TypeError):
        lib.grad_norm([g.half()])
    with pytest.raises(TypeError):
        lib.adamw_state_values([s])
    with pytest.raises(ValueError):
        lib.adamw_state(p, 16)
    lib.adamw_step([], [], [], 1, lr=1e-3)
    assert lib.adamw_state_values([]) == []


def test_offsets_beyond_32_bits(lib):
    """A tensor of more than 2^32 bytes and 2^31 entries: its last groups as the same entries by themselves."""
    n, m = 2 ** 31 + 700, 256 * 40 + 700 % 256
    g = gen(5)
    p, grad = (torch.zeros(n, dtype=BF16, device=DEV) for _ in range(2))
    p[-m:] = torch.randn(m, generator=g, device=DEV).bfloat16()
    grad[-m:] = torch.randn(m, generator=g, device=DEV).bfloat16()
    q, h = p[-m:].clone(), grad[-m:].clone()
    s, r = lib.adamw_state(p, 8), lib.adamw_state(q, 8)
    assert (n - m) % 256 == 0
    norm = lib.grad_norm([grad])
    assert abs(norm.item() - h.double().norm().item()) <= 1e-6 * norm.item()
    for k in (1, 2):
        lib.adamw_step([p], [grad], [s], k, grad_norm=norm, max_norm=1.0, **HYPER)
        lib.adamw_step([q], [h], [r], k, grad_norm=norm, max_norm=1.0, **HYPER)
    torch.cuda.synchronize()
    assert torch.equal(p[-m:], q) and not p[:-m].any()
    assert torch.equal(s["m"][-m:], r["m"]) and torch.equal(s["v"][-m:], r["v"]) and not s["v"][:-m].any()
    groups = r["m_scale"].numel()
    assert torch.equal(s["m_scale"][-groups:], r["m_scale"]) and torch.equal(s["v_scale"][-groups:], r["v_scale"])
    values = lib.adamw_state_values([s])[0]
    assert torch.equal(values["m"][-m:], lib.adamw_state_values([r])[0]["m"])
