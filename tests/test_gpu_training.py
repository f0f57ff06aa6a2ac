"""GPU parity of the training calls of the gated FFN with their formulas in 64 bits.  Run with `-m gpu` on a B200."""
import pytest
import torch

import training_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    yield m
    assert m.training_status(DEV) == 0


def make(T, D, H, dtype, seed, bias=True):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    rnd = lambda *shape, std=1.0: torch.randn(shape, generator=g, device=DEV) * std  # noqa: E731
    t = dict(x=rnd(T, D).to(dtype), W_g=rnd(H, D, std=D ** -0.5).to(dtype), W_up=rnd(H, D, std=D ** -0.5).to(dtype),
             W_down=rnd(H, D, std=D ** -0.5).to(dtype), b_g=rnd(H) - 0.8 if bias else None)
    t["dy"] = rnd(T, D).to(dtype)
    ld = (H + 7) // 8 * 8
    t["z"], t["u"] = (rnd(T, ld).to(dtype)[:, :H] for _ in range(2))
    return t


def check_forward(lib, t, act, act_up, what, **kw):
    bf16 = t["x"].dtype == torch.bfloat16
    w = [t[k] for k in ("x", "W_g", "b_g", "W_up", "W_down")]
    y, z, u = lib.gated_ffn_forward(*w, act, act_up, **kw)
    torch.cuda.synchronize()
    ref.assert_within(dict(y=y, z=z, u=u), ref.forward(*w, act, act_up), ref.forward_bounds(*w, act, act_up, bf16), what)
    return y, z, u


def check_backward(lib, t, act, act_up, what, **kw):
    bf16 = t["x"].dtype == torch.bfloat16
    w = [t[k] for k in ("dy", "x", "z", "u", "W_g", "W_up", "W_down")]
    got = lib.gated_ffn_backward(*w, act, act_up, **kw)
    torch.cuda.synchronize()
    want = {k: v for k, v in ref.backward(*w, act, act_up).items() if k in got}
    ref.assert_within(got, want, ref.backward_bounds(*w, act, act_up, bf16), what)
    return got


SHAPES = [(1, 8, 1), (1, 256, 1024), (2, 64, 7), (5, 72, 50), (64, 256, 1024), (63, 264, 129), (65, 64, 257), (127, 128, 128), (128, 520, 200),
          (129, 256, 1000), (257, 384, 511), (300, 200, 1531), (513, 136, 520), (3, 1096, 2057), (700, 328, 900)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D,H", SHAPES)
def test_forward_and_backward_at_odd_sizes(lib, T, D, H, dtype):
    t = make(T, D, H, dtype, 1000 * T + D + H)
    act, act_up = [("relu", None), ("sqrelu", "silu"), ("rsplus", "relu"), ("silu", None)][(T + D + H) % 4]
    check_forward(lib, t, act, act_up, f"forward {T}x{D}x{H} {act}/{act_up}")
    check_backward(lib, t, act, act_up, f"backward {T}x{D}x{H} {act}/{act_up}")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("act", ["relu", "sqrelu", "rsplus", "silu", "none"])
@pytest.mark.parametrize("act_up", [None, "relu", "sqrelu", "rsplus", "silu"])
def test_every_pair_of_activations(lib, act, act_up, dtype):
    t = make(70, 96, 150, dtype, 7, bias=act != "relu")
    check_forward(lib, t, act, act_up, f"{act}/{act_up}")
    check_backward(lib, t, act, act_up, f"{act}/{act_up}")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_a_wide_ffn_with_many_tokens(lib, dtype):
    t = make(1100, 1024, 2600, dtype, 3)
    check_forward(lib, t, "relu", None, "wide")
    check_backward(lib, t, "relu", None, "wide")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("T,D,H", [(300, 2048, 2045), (300, 2048, 2046), (300, 2048, 2047), (40, 2048, 4097), (520, 1032, 4099)])
def test_tiles_cut_along_k_with_hidden_widths_that_four_does_not_divide(lib, T, D, H, dtype):
    t = make(T, D, H, dtype, T + H)
    check_forward(lib, t, "sqrelu", "silu", f"forward {T}x{D}x{H}")
    check_backward(lib, t, "sqrelu", "silu", f"backward {T}x{D}x{H}")


def strided(t, extra, before):
    """The same values as rows of a wider matrix whose other columns hold a marker."""
    T, N = t.shape
    wide = torch.full((T, (N + 7) // 8 * 8 + extra), 77.0, dtype=t.dtype, device=t.device)
    wide[:, before:before + N] = t
    return wide[:, before:before + N], wide


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_strided_rows_and_untouched_columns(lib, dtype):
    T, D, H = 130, 136, 213
    t = make(T, D, H, dtype, 11)
    s = dict(t, x=strided(t["x"], 16, 8)[0], dy=strided(t["dy"], 24, 16)[0])
    outs = {k: strided(torch.zeros(T, n, dtype=dtype, device=DEV), 16, 8) for k, n in (("y", D), ("z", H), ("u", H), ("dx", D))}
    y, z, u = check_forward(lib, s, "sqrelu", None, "strided", y=outs["y"][0], z=outs["z"][0], u=outs["u"][0])
    plain = lib.gated_ffn_forward(t["x"], t["W_g"], t["b_g"], t["W_up"], t["W_down"], "sqrelu")
    assert all(torch.equal(a, b) for a, b in zip((y, z, u), plain))
    s.update(z=outs["z"][0], u=outs["u"][0])
    got = check_backward(lib, s, "sqrelu", None, "strided", out=dict(dx=outs["dx"][0]))
    want = lib.gated_ffn_backward(t["dy"], t["x"], plain[1], plain[2], t["W_g"], t["W_up"], t["W_down"], "sqrelu")
    assert all(torch.equal(got[k], want[k]) for k in want)
    for k, (view, whole) in outs.items():
        n = view.shape[1]
        assert (whole[:, :8] == 77).all() and (whole[:, 8 + n:] == 77).all(), k


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_gradients_left_out_and_no_tokens(lib, dtype):
    t = make(40, 64, 90, dtype, 5)
    w = [t[k] for k in ("dy", "x", "z", "u", "W_g", "W_up", "W_down")]
    every = lib.gated_ffn_backward(*w, "rsplus", "silu")
    for need in (["dx"], ["dW_g"], ["dW_up"], ["dW_down"], ["db_g"], ["dx", "db_g"], ["dW_up", "dW_down"], []):
        got = lib.gated_ffn_backward(*w, "rsplus", "silu", need=need)
        assert sorted(got) == sorted(need) and all(torch.equal(got[k], every[k]) for k in need), need
    y, z, u = lib.gated_ffn_forward(t["x"], t["W_g"], t["b_g"], t["W_up"], t["W_down"])
    alone, none, _ = lib.gated_ffn_forward(t["x"], t["W_g"], t["b_g"], t["W_up"], t["W_down"], save=False)
    assert torch.equal(y, alone) and none is None
    e = make(0, 64, 90, dtype, 5)
    y, z, u = lib.gated_ffn_forward(e["x"], e["W_g"], e["b_g"], e["W_up"], e["W_down"])
    assert y.shape == (0, 64) and z.shape == (0, 90)
    out = {k: torch.full((90, 64), 3.0, dtype=dtype, device=DEV) for k in ("dW_g", "dW_up", "dW_down")}
    got = lib.gated_ffn_backward(e["dy"], e["x"], z, u, e["W_g"], e["W_up"], e["W_down"], out=dict(out, db_g=torch.ones(90, device=DEV)))
    torch.cuda.synchronize()
    assert got["dx"].shape == (0, 64) and all((got[k] == 0).all() for k in ("dW_g", "dW_up", "dW_down", "db_g"))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_repeats_bitwise_on_other_streams_and_in_a_graph(lib, dtype):
    t = make(333, 264, 700, dtype, 9)
    f = [t[k] for k in ("x", "W_g", "b_g", "W_up", "W_down")]
    first = lib.gated_ffn_forward(*f)
    b = [t["dy"], t["x"], first[1], first[2], t["W_g"], t["W_up"], t["W_down"]]
    grads = lib.gated_ffn_backward(*b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for _ in range(3):
        again = lib.gated_ffn_forward(*f, stream=side)
        more = lib.gated_ffn_backward(*b, stream=side)
        side.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(first, again)) and all(torch.equal(grads[k], more[k]) for k in grads)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, z, u = lib.gated_ffn_forward(*f)
        g = lib.gated_ffn_backward(t["dy"], t["x"], z, u, t["W_g"], t["W_up"], t["W_down"])
    keep = t["x"].clone()
    t["x"].normal_()
    graph.replay()
    torch.cuda.synchronize()
    assert not torch.equal(y, first[0])
    t["x"].copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, first[0]) and all(torch.equal(g[k], grads[k]) for k in grads)


def test_gradients_against_differences_of_the_forward_pass(lib):
    """L = sum(dy . y) along a direction: (L(+e) - L(-e)) / 2 e differs from the gradient's product with the direction by e^2 times
    a third derivative (e = 2^-6, order one: 2e-4 of it) and by the forward pass's rounding over e (1e-6 / 0.016: 1e-4)."""
    t = make(33, 64, 120, torch.float32, 21)
    t = {k: v.contiguous() if v is not None else None for k, v in t.items()}
    names = dict(x="dx", W_g="dW_g", W_up="dW_up", W_down="dW_down", b_g="db_g")

    def loss(**over):
        a = dict(t, **over)
        y, z, u = lib.gated_ffn_forward(a["x"], a["W_g"], a["b_g"], a["W_up"], a["W_down"], "silu", "silu")
        return (y.double() * t["dy"].double()).sum().item(), z, u

    _, z, u = loss()
    grads = lib.gated_ffn_backward(t["dy"], t["x"], z, u, t["W_g"], t["W_up"], t["W_down"], "silu", "silu")
    g = torch.Generator(device=DEV)
    g.manual_seed(5)
    e = 2.0 ** -6
    for k, name in names.items():
        d = torch.randn(t[k].shape, generator=g, device=DEV) * t[k].std()
        d = d + grads[name] * (t[k].std() / grads[name].std())   # not orthogonal to the gradient
        up, down = loss(**{k: t[k] + e * d})[0], loss(**{k: t[k] - e * d})[0]
        want = (grads[name].double() * d.double()).sum().item()
        assert abs((up - down) / (2 * e) - want) <= 2e-3 * abs(want), (k, (up - down) / (2 * e), want)


def test_autograd_node(lib):
    t = make(24, 64, 96, torch.float32, 31)
    leaves = [t[k].clone().requires_grad_() for k in ("x", "W_g", "b_g", "W_up", "W_down")]
    y = lib.GatedFFNFunction.apply(leaves[0].view(4, 6, 64), *leaves[1:], "rsplus", "silu")
    y.backward(t["dy"].view(4, 6, 64))
    y0, z, u = lib.gated_ffn_forward(*[w.detach() for w in leaves], "rsplus", "silu")
    assert torch.equal(y.detach().view(24, 64), y0)
    got = lib.gated_ffn_backward(t["dy"], t["x"], z, u, t["W_g"], t["W_up"], t["W_down"], "rsplus", "silu")
    for w, k in zip(leaves, ("dx", "dW_g", "db_g", "dW_up", "dW_down")):
        assert torch.equal(w.grad, got[k]), k


def test_neurons_that_do_not_fire_and_values_far_out(lib):
    """A token that fires nothing, activations far from zero (exponentials that overflow), zeros exactly at the edge."""
    for dtype in (torch.float32, torch.bfloat16):
        t = make(20, 64, 80, dtype, 41)
        t["x"][3] = 0
        t["b_g"].fill_(-1.0)
        t["z"][0], t["z"][1], t["z"][2], t["z"][5] = 200.0, -200.0, 0.0, -0.0
        t["u"][0, :40], t["u"][1, 40:] = -150.0, 150.0
        for act, act_up in (("relu", None), ("rsplus", "silu"), ("silu", "rsplus"), ("sqrelu", "relu")):
            y, z, u = check_forward(lib, t, act, act_up, "far")
            if act != "silu":
                assert (y[3] == 0).all()
            check_backward(lib, t, act, act_up, "far")


def test_training_and_inference_agree(lib):
    """The weights of a trained block go to sparse_ffn_forward as they are."""
    t = make(3, 256, 1024, torch.bfloat16, 51)
    y, _, _ = lib.gated_ffn_forward(t["x"], t["W_g"], t["b_g"], t["W_up"], t["W_down"], "relu")
    ffn = lib.SparseFFN(256, 1024, torch.bfloat16, B_max=4)
    torch.cuda.synchronize()
    s = ffn.sparse_ffn_forward(t["x"], {"W_g": t["W_g"]}, t["b_g"], t["W_up"], t["W_down"], "relu")
    torch.cuda.synchronize()
    assert (y.double() - s.double()).norm() <= 1e-2 * s.double().norm()


def test_refusals(lib):
    t = make(16, 64, 40, torch.bfloat16, 61)
    f = [t[k] for k in ("x", "W_g", "b_g", "W_up", "W_down")]
    b = [t[k] for k in ("dy", "x", "z", "u", "W_g", "W_up", "W_down")]
    with pytest.raises(TypeError):
        lib.gated_ffn_forward(t["x"].float(), *f[1:])
    with pytest.raises(TypeError):
        lib.gated_ffn_forward(t["x"].cpu(), *f[1:])
    with pytest.raises(TypeError):
        lib.gated_ffn_forward(t["x"], t["W_g"].half(), *f[2:])
    with pytest.raises(TypeError):
        lib.gated_ffn_forward(t["x"], t["W_g"].T.contiguous().T, *f[2:])
    with pytest.raises(TypeError):
        lib.gated_ffn_forward(t["x"], t["W_g"], t["b_g"].bfloat16(), *f[3:])
    with pytest.raises(KeyError):
        lib.gated_ffn_forward(*f, "gelu")
    with pytest.raises(lib.SFFNError) as err:                                # rows that are no multiple of 16 bytes
        lib.gated_ffn_forward(torch.zeros(16, 66, dtype=torch.bfloat16, device=DEV)[:, :64], *f[1:])
    assert err.value.code == 2
    with pytest.raises(lib.SFFNError) as err:
        lib.gated_ffn_forward(t["x"][:, :60].contiguous(), *[w[:, :60].contiguous() if w.dim() == 2 else w for w in f[1:]])
    assert err.value.code == 2
    with pytest.raises(lib.SFFNError) as err:                                # not on 16 bytes
        lib.gated_ffn_forward(torch.zeros(16 * 64 + 1, dtype=torch.bfloat16, device=DEV)[1:].view(16, 64), *f[1:])
    assert err.value.code == 2
    with pytest.raises(ValueError):
        lib.gated_ffn_backward(*b, need=["dV"])
    with pytest.raises(TypeError):
        lib.gated_ffn_backward(*b, out=dict(dW_g=torch.zeros(40, 64, device=DEV)))
    with pytest.raises(TypeError):
        lib.gated_ffn_backward(b[0], b[1], t["z"], torch.zeros(16, 48, dtype=torch.bfloat16, device=DEV)[:, :40], *b[4:])

def test_offsets_beyond_32_bits(lib):
    """z and u of more than 2^31 entries: the last rows against the same rows by themselves."""
    T, D, H = 150_001, 64, 14336
    g = torch.Generator(device=DEV)
    g.manual_seed(71)
    x = torch.randn(T, D, generator=g, device=DEV).bfloat16()
    W = [(torch.randn(H, D, generator=g, device=DEV) * D ** -0.5).bfloat16() for _ in range(3)]
    b_g = torch.randn(H, generator=g, device=DEV)
    y, z, u = lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2])
    n = 300
    y1, z1, u1 = lib.gated_ffn_forward(x[-n:], W[0], b_g, W[1], W[2])
    torch.cuda.synchronize()
    assert z.numel() > 2 ** 31
    # tiles lie differently over the rows, and a tile may be cut along K (64 here: it is not): the same sums
    assert torch.equal(z[-n:], z1) and torch.equal(u[-n:], u1)
    assert (y[-n:].double() - y1.double()).abs().max() <= 2 ** -7 * y1.double().abs().max()
    dy = torch.zeros(T, D, device=DEV, dtype=torch.bfloat16)
    dy[-n:] = torch.randn(n, D, generator=g, device=DEV)
    got = lib.gated_ffn_backward(dy, x, z, u, *W)                      # rows without a gradient add nothing
    want = lib.gated_ffn_backward(dy[-n:], x[-n:], z1, u1, *W)
    assert (got["dx"][:-n] == 0).all()
    for k in ("dx", "dW_g", "dW_up", "dW_down", "db_g"):
        a, b = got[k][-n:] if k == "dx" else got[k], want[k]
        assert (a.double() - b.double()).norm() <= 2 ** -8 * b.double().norm(), k
