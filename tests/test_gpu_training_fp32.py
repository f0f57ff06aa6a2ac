"""fp32 training calls past the size from which they run on the tensor cores, and over widths that four divides and eight does not: strides,
alignments, pairs of activations, outputs left out, streams and graphs.  Run with `-m gpu` on a B200."""
import pytest
import torch

import training_reference as ref
from test_gpu_training import check_backward, check_forward, make

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32 = torch.float32
BIG = (300, 1028, 1027)     # 3.2e8 products: on the tensor cores, forward and backward


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    yield m
    assert m.training_status(DEV) == 0


def placed(t, offset, extra):
    """The same values as rows of a wider matrix that starts `offset` entries into its buffer, all else 77; the matrix and the buffer."""
    T, N = t.shape
    ld = (N + 3) // 4 * 4 + extra
    buffer = torch.full((T * ld + offset + 8,), 77.0, dtype=t.dtype, device=DEV)
    view = buffer[offset:offset + T * ld].view(T, ld)[:, :N]
    view.copy_(t)
    return view, buffer


def untouched(view, buffer):
    mask = torch.ones_like(buffer, dtype=torch.bool)
    mask[view.storage_offset():view.storage_offset() + view.stride(0) * view.shape[0]].view(view.shape[0], -1)[:, :view.shape[1]] = False
    return bool((buffer[mask] == 77).all())


@pytest.mark.parametrize("T", [1, 5, 16, 17, 40, 300])
@pytest.mark.parametrize("D,H", [(12, 50), (260, 129), (1028, 1027)])
def test_widths_that_four_divides(lib, T, D, H):
    """Plain, and with x, dy, y, z, u and dx on 16 bytes but not on 32, rows 16 bytes more than their width apart."""
    t = make(T, D, H, F32, T + D)
    t["z"], t["u"] = (torch.randn(T, (H + 3) // 4 * 4, device=DEV)[:, :H] for _ in range(2))
    act, act_up = [("relu", None), ("sqrelu", "silu"), ("rsplus", "relu")][(T + D) % 3]
    y, z, u = check_forward(lib, t, act, act_up, f"{T}x{D}x{H}")
    grads = check_backward(lib, t, act, act_up, f"{T}x{D}x{H}")
    s = dict(t, **{k: placed(t[k], 4, 4)[0] for k in ("x", "dy", "z", "u")})
    outs = {k: placed(torch.zeros(T, n, device=DEV), 4, 4) for k, n in (("y", D), ("z", H), ("u", H), ("dx", D))}
    got = lib.gated_ffn_forward(s["x"], t["W_g"], t["b_g"], t["W_up"], t["W_down"], act, act_up, y=outs["y"][0], z=outs["z"][0], u=outs["u"][0])
    assert all(torch.equal(a, b) for a, b in zip(got, (y, z, u)))
    more = lib.gated_ffn_backward(s["dy"], s["x"], s["z"], s["u"], t["W_g"], t["W_up"], t["W_down"], act, act_up, out=dict(dx=outs["dx"][0]))
    assert all(torch.equal(more[k], grads[k]) for k in grads)
    assert all(untouched(*o) for o in outs.values())


@pytest.mark.parametrize("H", [1024, 1025, 1026, 1027, 1028, 1030])
def test_hidden_widths_and_rows_on_either_alignment(lib, H):
    """On the tensor cores: z, u and outputs whose rows start on 32 bytes, and on 16 only."""
    T, D = 300, 1032
    t = make(T, D, H, F32, H)
    y, z, u = check_forward(lib, t, "sqrelu", None, f"H {H}")
    grads = check_backward(lib, t, "sqrelu", None, f"H {H}")
    for offset in (0, 4, 8):
        for extra in (0, 4, 8):
            outs = {k: placed(torch.zeros(T, n, device=DEV), offset, extra) for k, n in (("y", D), ("z", H), ("u", H), ("dx", D))}
            got = lib.gated_ffn_forward(t["x"], t["W_g"], t["b_g"], t["W_up"], t["W_down"], "sqrelu", y=outs["y"][0], z=outs["z"][0], u=outs["u"][0])
            assert all(torch.equal(a, b) for a, b in zip(got, (y, z, u))), (offset, extra)
            zin, uin = placed(t["z"], offset, extra)[0], placed(t["u"], offset, extra)[0]
            more = lib.gated_ffn_backward(t["dy"], t["x"], zin, uin, t["W_g"], t["W_up"], t["W_down"], "sqrelu", out=dict(dx=outs["dx"][0]))
            assert all(torch.equal(more[k], grads[k]) for k in grads), (offset, extra)
            assert all(untouched(*o) for o in outs.values()), (offset, extra)


@pytest.mark.parametrize("act", ["relu", "sqrelu", "rsplus", "silu", "none"])
@pytest.mark.parametrize("act_up", [None, "relu", "sqrelu", "rsplus", "silu"])
def test_every_pair_of_activations(lib, act, act_up):
    t = make(*BIG, F32, 7, bias=act != "relu")
    check_forward(lib, t, act, act_up, f"{act}/{act_up}")
    check_backward(lib, t, act, act_up, f"{act}/{act_up}")


def test_gradients_left_out_and_nothing_saved(lib):
    t = make(*BIG, F32, 5)
    w = [t[k] for k in ("dy", "x", "z", "u", "W_g", "W_up", "W_down")]
    for need in (["dx"], ["dW_g"], ["dW_up"], ["dW_down"], ["db_g"], ["dx", "db_g"], ["dW_up", "dW_down"], []):
        got = check_backward(lib, t, "rsplus", "silu", str(need), need=need)     # bits follow from which outputs are asked for
        again = lib.gated_ffn_backward(*w, "rsplus", "silu", need=need)
        assert sorted(got) == sorted(need) and all(torch.equal(got[k], again[k]) for k in need), need
    f = [t[k] for k in ("x", "W_g", "b_g", "W_up", "W_down")]
    y, z, u = lib.gated_ffn_forward(*f)
    alone, none, _ = lib.gated_ffn_forward(*f, save=False)
    assert torch.equal(y, alone) and none is None


def test_values_far_out(lib):
    """Exponentials that overflow, zeros at the edge, a token that fires nothing, entries of 1e-30 and 1e30 (whose terms are far apart)."""
    t = make(*BIG, F32, 41)
    t["x"][3] = 0
    t["x"][7, :9], t["x"][8, :9] = 1e-30, 1e6
    t["b_g"].fill_(-1.0)
    t["z"][0], t["z"][1], t["z"][2], t["z"][5] = 200.0, -200.0, 0.0, -0.0
    t["u"][0, :40], t["u"][1, 40:] = -150.0, 150.0
    for act, act_up in (("relu", None), ("rsplus", "silu"), ("silu", "rsplus"), ("sqrelu", "relu")):
        y, _, _ = check_forward(lib, t, act, act_up, "far")
        if act != "silu":
            assert (y[3] == 0).all()
        check_backward(lib, t, act, act_up, "far")


def test_repeats_bitwise_on_other_streams_and_in_a_graph(lib):
    t = make(*BIG, F32, 9)
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
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, first[0]) and all(torch.equal(g[k], grads[k]) for k in grads)


@pytest.mark.parametrize("dtype", [F32, torch.bfloat16], ids=["f32", "bf16"])
def test_autograd_node_with_frozen_weights(lib, dtype):
    t = make(*(BIG if dtype == F32 else (300, 264, 130)), dtype, 31)
    D = t["x"].shape[1]
    for wanted in ((True,) * 5, (False, True, True, False, True), (True, False, False, False, False)):
        leaves = [t[k].clone().requires_grad_(w) for k, w in zip(("x", "W_g", "b_g", "W_up", "W_down"), wanted)]
        y = lib.GatedFFNFunction.apply(leaves[0].view(3, 100, D), *leaves[1:], "rsplus", "silu")
        y.backward(t["dy"].view(3, 100, D))
        _, z, u = lib.gated_ffn_forward(*[w.detach() for w in leaves], "rsplus", "silu")
        names = ("dx", "dW_g", "db_g", "dW_up", "dW_down")
        got = lib.gated_ffn_backward(t["dy"], t["x"], z, u, t["W_g"], t["W_up"], t["W_down"], "rsplus", "silu", need=[n for n, w in zip(names, wanted) if w])
        for w, wants, k in zip(leaves, wanted, names):
            assert torch.equal(w.grad, got[k]) if wants else w.grad is None, k
