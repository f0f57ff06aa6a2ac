"""The norms around a block over many rows, which come through shared memory, and at values, strides and alignments where that can go
wrong.  Run with `-m gpu` on a B200."""
import pytest
import torch

import block_reference as ref
from test_gpu_block_norm import BF16, DEV, F32, IDS, TYPES, both, check_backward, check_forward, inputs, lib, rand, gen  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("types", TYPES, ids=IDS)
@pytest.mark.parametrize("T,D", [(1300, 1032), (1184, 2048), (1190, 2056), (1200, 4104), (1187, 8192), (1500, 1160)])
def test_many_rows(lib, T, D, types):  # noqa: F811
    both(lib, T, D, types, "channel", True, True, seed=T)


@pytest.mark.parametrize("types", [TYPES[0], TYPES[1], TYPES[3]], ids=[IDS[0], IDS[1], IDS[3]])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
@pytest.mark.parametrize("post,pre", [(True, True), (True, False), (False, True), (False, False)])
def test_kinds_over_many_rows(lib, types, gate, post, pre):  # noqa: F811
    both(lib, 1250, 1064, types, gate, post, pre)


def test_widths_that_eight_does_not_divide(lib):  # noqa: F811
    for D in (1028, 2052, 4100, 8188):
        both(lib, 1184, D, TYPES[0], "full", True, True, seed=D)


@pytest.mark.parametrize("T", [7, 1300])
@pytest.mark.parametrize("extra", [4, 8, 12])
def test_fp32_rows_on_sixteen_bytes_only(lib, T, extra):  # noqa: F811
    """Strides that are a multiple of 16 bytes, not of 32, and bases likewise; h over resid, dresid over dh; nothing between rows is written."""
    D = 1100
    c, dh, dn = inputs(T, D, TYPES[0], "full", True, True)
    want = lib.block_norm_forward(**c)
    back = (dh, dn, c["y"], want[0], want[2], c["post_gain"], c["pre_gain"], c["gate"])
    grads = lib.block_norm_backward(*back)

    def apart(t):
        room = torch.full((T + 1, D + extra), 77.0, device=DEV)
        at = room.view(-1)[4:4 + T * (D + extra)].view(T, D + extra)[:, :D]
        at.copy_(t)
        return room, at

    rooms = {k: apart(c[k]) for k in ("y", "resid", "gate")}
    n_room, n = apart(c["y"])
    x = rooms["resid"][1]
    got = lib.block_norm_forward(rooms["y"][1], x, c["post_gain"], c["pre_gain"], rooms["gate"][1], h=x, n=n)
    assert torch.equal(x, want[0]) and torch.equal(n, want[1]) and torch.equal(got[2], want[2])
    a_room, a = apart(dh)
    d_room, d = apart(c["gate"])
    y_room, y = apart(c["y"])
    got = lib.block_norm_backward(a, apart(dn)[1], rooms["y"][1], x, want[2], c["post_gain"], c["pre_gain"], rooms["gate"][1], out=dict(dresid=a, dy=y, dgate=d))
    for k in grads:
        assert torch.equal(got[k], grads[k]), k
    for room in (rooms["resid"][0], n_room, a_room, d_room, y_room):
        left = room.view(-1)
        assert (left[:4] == 77).all() and (left[4:4 + T * (D + extra)].view(T, -1)[:, D:] == 77).all() and (left[4 + T * (D + extra):] == 77).all()


@pytest.mark.parametrize("size", [1e-15, 1e-10, 1e10, 1e15])
def test_gradients_of_small_and_large_rows(lib, size):  # noqa: F811
    """The cube of a row's statistic leaves fp32 where the gradient does not.  eps is zero: beside 1e-15 it would be all there is."""
    c, dh, dn = inputs(30, 264, TYPES[0], "none", True, True)
    c["y"] *= size
    c["resid"] *= size
    h, n, stats = lib.block_norm_forward(**c, scale=size, eps=0.0)
    check_forward(c, (h, n, stats), size, 0.0)
    args = (dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], None)
    check_backward(args, lib.block_norm_backward(*args, scale=size), size)


def test_same_bits_and_a_graph_over_many_rows(lib):  # noqa: F811
    c, dh, dn = inputs(1400, 2056, TYPES[1], "token", True, True)
    gains = (c["post_gain"], c["pre_gain"], c["gate"])
    h, n, stats = lib.block_norm_forward(**c)
    want = lib.block_norm_backward(dh, dn, c["y"], h, stats, *gains)
    for _ in range(3):
        h2, n2, stats2 = lib.block_norm_forward(**c)
        got = lib.block_norm_backward(dh, dn, c["y"], h2, stats2, *gains)
        assert torch.equal(h, h2) and torch.equal(n, n2) and torch.equal(stats, stats2) and all(torch.equal(got[k], want[k]) for k in want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h3, n3, stats3 = lib.block_norm_forward(**c)
        got = lib.block_norm_backward(dh, dn, c["y"], h3, stats3, *gains)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, h3) and torch.equal(n, n3) and all(torch.equal(got[k], want[k]) for k in want)


def test_two_streams_at_once(lib):  # noqa: F811
    """Calls that overlap have nothing in common."""
    sides = [torch.cuda.Stream() for _ in range(2)]
    sets = [inputs(1400, 4096, TYPES[1], "channel", True, True, seed=s) for s in range(2)]
    want = []
    for c, dh, dn in sets:
        h, n, stats = lib.block_norm_forward(**c)
        want.append((h, n, lib.block_norm_backward(dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], c["gate"])))
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for side, (c, dh, dn), out in zip(sides, sets, got):
            h, n, stats = lib.block_norm_forward(**c, stream=side)
            out.append((h, n, lib.block_norm_backward(dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], c["gate"], stream=side)))
    torch.cuda.synchronize()
    for a, outs in zip(want, got):
        for b in outs:
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and all(torch.equal(a[2][k], b[2][k]) for k in a[2])


def test_a_graph_node_in_a_captured_backward_pass(lib):  # noqa: F811
    """Forward and backward pass of the node in one graph.  (Leaves of its own: torch itself cannot capture a backward pass while an eager
    graph of the same leaves lives, whatever its nodes are.)"""
    c, a, b = inputs(40, 128, TYPES[1], "channel", True, True)
    names = ("y", "resid", "post_gain", "pre_gain", "gate")

    def run():
        args = [c[k].clone().requires_grad_() for k in names]
        h, n = lib.BlockNormFunction.apply(*args)
        return torch.autograd.grad([(h * a).sum() + (n * b).sum()], args)

    want = run()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = run()
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)
