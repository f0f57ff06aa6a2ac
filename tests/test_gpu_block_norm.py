"""GPU parity of the norms around a block with their formulas in 64 bits.  Run with `-m gpu` on a B200."""
import pytest
import torch

import block_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
TYPES = [(F32, F32, F32), (BF16, BF16, BF16), (F32, BF16, BF16), (BF16, F32, BF16), (BF16, BF16, F32), (F32, F32, BF16)]
IDS = ["-".join("f32" if t is F32 else "bf16" for t in c) for c in TYPES]


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    return m


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rand(shape, dtype, g, std=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def inputs(T, D, types, gate, post, pre, seed=0):
    g = gen(seed)
    ty, th, tn = types
    c = dict(y=rand((T, D), ty, g, 0.5), resid=rand((T, D), th, g, 2.0))
    c["post_gain"] = 1 + rand((D,), F32, g, 0.3) if post else None
    c["pre_gain"] = 1 + rand((D,), F32, g, 0.3) if pre else None
    shape = dict(none=None, channel=(D,), token=(T, 1), full=(T, D))[gate]
    c["gate"] = None if shape is None else rand(shape, th if gate == "full" else F32, g)
    return c, rand((T, D), th, g), rand((T, D), tn, g) if pre else None


def check_forward(c, got, scale, eps):
    want, size = ref.forward(*[c[k] for k in ("y", "resid", "post_gain", "pre_gain", "gate")], scale, eps)
    h, n, stats = got
    ref.close("h", h, want["h"], size["h"], ref.ROW)
    if c["pre_gain"] is not None:
        ref.close("n", n, want["n"], size["n"], ref.ROW)
    else:
        assert n is None
    if stats is not None:
        ref.close("r", stats[0], want["stats"][0], want["stats"][0], ref.ROW)
        if c["pre_gain"] is not None:  # of h before it is rounded; its terms may cancel
            rho = want["stats"][1]
            ref.close("rho", stats[1], rho, rho + rho ** 3 * (want["h"].abs() * size["h"]).mean(1), ref.ROW)
        else:
            assert not stats[1].any()


def check_backward(args, got, scale):
    want, size = ref.backward(*args, scale)
    assert got.keys() == want.keys()
    T = args[3].shape[0]
    for k in want:
        ref.close(k, got[k], want[k], size[k], ref.column(T) if k in ("dpost_gain", "dpre_gain") or (k == "dgate" and got[k].dim() == 1) else ref.ROW)


def both(lib, T, D, types, gate, post, pre, scale=0.7, eps=1e-5, seed=0):
    c, dh, dn = inputs(T, D, types, gate, post, pre, seed)
    h, n, stats = lib.block_norm_forward(**c, scale=scale, eps=eps, n_dtype=types[2])
    assert h.dtype == types[1] and (n is None or n.dtype == types[2])
    check_forward(c, (h, n, stats), scale, eps)
    args = (dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], c["gate"])
    check_backward(args, lib.block_norm_backward(*args, scale=scale), scale)


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_kinds(lib, types, gate, post, pre):
    both(lib, 37, 264, types, gate, post, pre)
    both(lib, 3, 2056, types, gate, post, pre, seed=1)


@pytest.mark.parametrize("T,D", [(1, 8), (1, 64), (2, 256), (9, 264), (1, 512), (700, 512), (5, 520), (3, 1024), (300, 1024), (5, 1032), (1, 2048), (400, 2048),
                                 (3, 2056), (1, 4096), (333, 4096), (2, 4104), (1, 8192), (200, 8192), (3, 8200), (2, 16384), (3, 16392), (2, 32768), (5000, 64),
                                 (2500, 200)])
def test_sizes(lib, T, D):
    for types in (TYPES[0], TYPES[1], TYPES[2]):
        both(lib, T, D, types, "channel", True, True, seed=T + D)


@pytest.mark.parametrize("D", [4, 12, 60, 260, 1028])
def test_widths_of_fp32_that_eight_does_not_divide(lib, D):
    for gate in ("none", "channel", "token", "full"):
        both(lib, 21, D, TYPES[0], gate, True, True)


def test_no_tokens(lib):
    c, dh, dn = inputs(0, 64, TYPES[1], "channel", True, True)
    h, n, stats = lib.block_norm_forward(**c)
    assert h.shape == n.shape == (0, 64) and stats.shape == (2, 0)
    got = lib.block_norm_backward(dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], c["gate"])
    for k in ("dpost_gain", "dpre_gain", "dgate"):
        assert got[k].shape == (64,) and not got[k].any()


@pytest.mark.parametrize("types", [TYPES[0], TYPES[1]], ids=["f32", "bf16"])
def test_parts_left_out(lib, types):
    T, D = 50, 320
    c, dh, dn = inputs(T, D, types, "none", True, True)
    # only a norm: h is resid
    h, n, stats = lib.block_norm_forward(None, c["resid"], None, c["pre_gain"])
    assert h is c["resid"]
    check_forward(dict(c, y=None, post_gain=None), (h, n, stats), 1.0, 1e-6)
    args = (dh, dn, None, h, stats, None, c["pre_gain"], None)
    check_backward(args, lib.block_norm_backward(*args), 1.0)
    # no stream
    h, n, stats = lib.block_norm_forward(c["y"], None, c["post_gain"], c["pre_gain"], scale=2.0)
    check_forward(dict(c, resid=None), (h, n, stats), 2.0, 1e-6)
    # one of the gradients that come in
    for a, b in ((dh, None), (None, dn)):
        args = (a, b, c["y"], h, stats, c["post_gain"], c["pre_gain"], None)
        check_backward(args, lib.block_norm_backward(*args, scale=2.0), 2.0)
    # a part of what comes out, and nothing saved
    whole = lib.block_norm_backward(dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], None)
    for k in whole:
        got = lib.block_norm_backward(dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], None, need=(k,))
        assert list(got) == [k] and torch.equal(got[k], whole[k])
    assert lib.block_norm_forward(c["y"], c["resid"], c["post_gain"], save=False)[1:] == (None, None)


def test_one_token_without_rows(lib):
    c, dh, dn = inputs(1, 256, TYPES[2], "channel", True, True)
    h, n, stats = lib.block_norm_forward(c["y"][0], c["resid"][0], c["post_gain"], c["pre_gain"], c["gate"], n_dtype=BF16)
    h2, n2, stats2 = lib.block_norm_forward(**c, n_dtype=BF16)
    assert h.shape == (256,) and torch.equal(h, h2[0]) and torch.equal(n, n2[0])
    got = lib.block_norm_backward(dh[0], dn[0], c["y"][0], h, stats, c["post_gain"], c["pre_gain"], c["gate"])
    want = lib.block_norm_backward(dh, dn, c["y"], h2, stats2, c["post_gain"], c["pre_gain"], c["gate"])
    for k in want:
        assert torch.equal(got[k], want[k].view(got[k].shape)), k


def test_rows_apart_in_place_and_what_lies_between(lib):
    """Strided inputs and outputs; between the rows, and behind the last one, nothing is written."""
    T, D = 40, 264
    c, dh, dn = inputs(T, D, TYPES[1], "full", True, True)
    want_h, want_n, want_stats = lib.block_norm_forward(**c)

    def apart(t, extra):
        room = torch.full((T + 2, D + extra), 77.0, dtype=t.dtype, device=DEV)
        room[1:-1, :D] = t
        return room, room[1:-1, :D]

    def between(room):
        return bool((room[:, D:] == 77).all() and (room[0] == 77).all() and (room[-1] == 77).all())

    s = {k: apart(c[k], e)[1] for k, e in (("y", 8), ("resid", 24), ("gate", 16))}
    (hr, h), (nr, n) = apart(c["y"], 40), apart(c["y"], 8)
    got = lib.block_norm_forward(s["y"], s["resid"], c["post_gain"], c["pre_gain"], s["gate"], h=h, n=n)
    assert got[0] is not None and torch.equal(h, want_h) and torch.equal(n, want_n) and torch.equal(got[2], want_stats) and between(hr) and between(nr)
    room, x = apart(c["resid"], 8)
    lib.block_norm_forward(s["y"], x, c["post_gain"], c["pre_gain"], s["gate"], h=x)
    assert torch.equal(x, want_h) and between(room)
    want = lib.block_norm_backward(dh, dn, c["y"], want_h, want_stats, c["post_gain"], c["pre_gain"], c["gate"])
    (ar, a), (br, b), (gr, g) = apart(dh, 16), apart(dh, 8), apart(dh, 24)
    got = lib.block_norm_backward(a, apart(dn, 8)[1], s["y"], h, want_stats, c["post_gain"], c["pre_gain"], s["gate"], out=dict(dresid=a, dy=b, dgate=g))
    for k in want:
        assert torch.equal(got[k], want[k]), k
    assert between(ar) and between(br) and between(gr) and got["dresid"].data_ptr() == a.data_ptr()


def test_small_and_large_values(lib):
    """Rows of zeros (the statistic is 1 / sqrt(eps)), tiny rows, rows whose squares are near the end of fp32, and a row with a NaN, which
    stays in its row but for the columns' sums."""
    T, D = 8, 256
    c, dh, dn = inputs(T, D, TYPES[0], "none", True, True)
    c["y"][0] = 0
    c["resid"][0] = 0
    c["y"][1] *= 1e-18
    c["y"][2] *= 1e17
    h, n, stats = lib.block_norm_forward(**c, eps=1e-6)
    check_forward(c, (h, n, stats), 1.0, 1e-6)
    assert not h[0].any() and not n[0].any() and abs(stats[0, 0].item() - 1000) < 0.01
    got = lib.block_norm_backward(dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], None)
    assert all(torch.isfinite(t).all() for t in got.values())
    c["y"][4, 17] = float("nan")
    h2, n2, _ = lib.block_norm_forward(**c, eps=1e-6)
    keep = [i for i in range(T) if i != 4]
    assert torch.equal(h2[keep], h[keep]) and torch.equal(n2[keep], n[keep]) and n2[4].isnan().all()


def test_same_bits_other_streams_and_a_graph(lib):
    T, D = 500, 1032
    c, dh, dn = inputs(T, D, TYPES[1], "channel", True, True)
    gains = (c["post_gain"], c["pre_gain"], c["gate"])
    h, n, stats = lib.block_norm_forward(**c)
    want = lib.block_norm_backward(dh, dn, c["y"], h, stats, *gains)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        h2, n2, stats2 = lib.block_norm_forward(**c, stream=side)
        got = lib.block_norm_backward(dh, dn, c["y"], h2, stats2, *gains, stream=side)
        side.synchronize()
        assert torch.equal(h, h2) and torch.equal(n, n2) and all(torch.equal(got[k], want[k]) for k in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h3, n3, stats3 = lib.block_norm_forward(**c)
        got = lib.block_norm_backward(dh, dn, c["y"], h3, stats3, *gains)
    c["y"].copy_(rand((T, D), BF16, gen(9)))
    h, n, stats = lib.block_norm_forward(**c)
    want = lib.block_norm_backward(dh, dn, c["y"], h, stats, *gains)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, h3) and torch.equal(n, n3) and all(torch.equal(got[k], want[k]) for k in want)


def test_offsets_beyond_32_bits(lib):
    """Rows so far apart that the last one starts beyond 2^32 elements."""
    T, D, ld = 3, 64, (1 << 31) - 64
    room = torch.zeros((T - 1) * ld + D, dtype=BF16, device=DEV)
    far = room.as_strided((T, D), (ld, 1))
    c, dh, dn = inputs(T, D, TYPES[1], "none", True, True)
    far.copy_(c["y"])
    a, b = lib.block_norm_forward(**c), lib.block_norm_forward(far, c["resid"], c["post_gain"], c["pre_gain"])
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    x = lib.block_norm_backward(dh, dn, c["y"], a[0], a[2], c["post_gain"], c["pre_gain"])
    lib.block_norm_backward(dh, dn, c["y"], a[0], a[2], c["post_gain"], c["pre_gain"], need=("dresid",), out=dict(dresid=far))
    assert torch.equal(far, x["dresid"])


@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
def test_graph_node_against_differences(lib, gate):
    """The node's gradients against differences of the 64-bit forward pass along random directions, in fp32: a central difference of step
    e is off by e^2 times a third derivative; the gradients by ROW units of their terms' size, far below 1e-3 of the whole."""
    c, a, b = inputs(12, 64, TYPES[0], gate, True, True)
    leaves = {k: v.clone().requires_grad_() for k, v in c.items() if v is not None}
    args = [leaves.get(k) for k in ("y", "resid", "post_gain", "pre_gain", "gate")]
    h, n = lib.BlockNormFunction.apply(*args, 0.7, 1e-5)
    ((h * a).sum() + (n * b).sum()).backward()

    def loss(values):
        out, _ = ref.forward(*[values.get(k) for k in ("y", "resid", "post_gain", "pre_gain", "gate")], 0.7, 1e-5)
        return ((out["h"] * a.double()).sum() + (out["n"] * b.double()).sum()).item()

    g = gen(5)
    for k, leaf in leaves.items():
        way = torch.randn(leaf.shape, generator=g, device=DEV, dtype=torch.float64)
        e = 1e-5
        up, down = ({q: v.detach().double() + (s * e * way if q == k else 0) for q, v in leaves.items()} for s in (1, -1))
        slope = (loss(up) - loss(down)) / (2 * e)
        got = (leaf.grad.double() * way).sum().item()
        size = (leaf.grad.double() * way).abs().sum().item()
        assert abs(got - slope) <= 1e-4 * size, (k, got, slope)


def test_graph_node_parts(lib):
    """Three dimensions, an output that nothing uses, leaves that need no gradient, and no second derivative."""
    g = gen(3)
    y, x = rand((2, 5, 64), BF16, g).requires_grad_(), rand((2, 5, 64), BF16, g)
    gain, token = torch.ones(64, device=DEV), rand((2, 5, 1), F32, g).requires_grad_()
    h, n = lib.BlockNormFunction.apply(y, x, gain, gain, token)
    assert h.shape == n.shape == (2, 5, 64)
    h.sum().backward()
    assert y.grad.shape == y.shape and token.grad.shape == token.shape and x.grad is None
    first = y.grad.clone()
    h, n = lib.BlockNormFunction.apply(y, x, gain, None, token)
    assert n is None
    y.grad = None
    h.sum().backward()
    assert torch.equal(y.grad, first)
    x = x.clone().requires_grad_()
    h, n = lib.BlockNormFunction.apply(None, x, None, gain)
    n.sum().backward()
    assert x.grad is not None and torch.equal(h, x)
    h, n = lib.BlockNormFunction.apply(y, x, gain, gain, token)
    (gx,) = torch.autograd.grad(n.float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        gx.sum().backward()
    h, n = lib.BlockNormFunction.apply(y, x, gain, gain, token)
    with torch.no_grad():
        h.add_(1)
    with pytest.raises(RuntimeError):  # h was saved
        n.sum().backward()


def test_refusals(lib):
    c, dh, dn = inputs(4, 64, TYPES[1], "channel", True, True)
    h, n, stats = lib.block_norm_forward(**c)
    for bad in (dict(y=None, resid=None), dict(y=c["y"].cpu()), dict(y=c["y"].half()), dict(post_gain=c["post_gain"][:32]), dict(post_gain=c["post_gain"].bfloat16()),
                dict(gate=c["gate"][None].expand(4, 64)), dict(gate=c["gate"][:, None]), dict(resid=c["resid"][:3]), dict(h=n.float()), dict(n_dtype=torch.float16),
                dict(resid=c["resid"].t().contiguous().t()), dict(y=None, h=h), dict(pre_gain=None, n=n)):
        with pytest.raises(TypeError):
            lib.block_norm_forward(**{**c, **bad})
    for bad in (dict(n=c["y"]), dict(n=c["resid"]), dict(h=c["y"]), dict(h=n, n=n), dict(y=None), dict(scale=float("inf")), dict(eps=-1.0), dict(y=dh[:, :60], resid=dn[:, :60], gate=None)):
        with pytest.raises((lib.SFFNError, TypeError)):
            lib.block_norm_forward(**{**c, **bad})
    args = (dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], c["gate"])
    for bad in (dict(need=("dx",)), dict(out=dict(dx=dh))):
        with pytest.raises(ValueError):
            lib.block_norm_backward(*args, **bad)
    for out in (dict(dy=dn), dict(dy=dh), dict(dresid=dn), dict(dresid=c["y"]), dict(dpre_gain=c["pre_gain"]), dict(dgate=c["gate"])):
        with pytest.raises(lib.SFFNError):
            lib.block_norm_backward(*args, out=out)
    with pytest.raises(ValueError):
        lib.block_norm_backward(None, None, *args[2:])
    assert all(torch.equal(a, b) for a, b in zip(lib.block_norm_forward(**c), (h, n, stats)))
