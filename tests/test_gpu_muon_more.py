"""Muon and the orthogonalised update in company: two calls at once, a model's step with everything in one stream, serving after a step, and the
sizes at which products change their form.  Run with `-m gpu` on a B200."""
import pytest
import torch

import muon_reference as ref
from test_gpu_muon import BF16, DEV, F32, STEP, check_step, copy, gen, lib, normal, tensors  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("shape", [(128, 128), (129, 200), (700, 600), (720, 600), (900, 600), (1030, 1024), (1536, 1024), (1540, 1028), (2300, 1800), (3000, 2100), (300, 20000),
                                   (20000, 300), (40, 100000), (2049, 2047)], ids=str)
def test_where_products_change_form(lib, shape, bits):  # noqa: F811
    """One, two and three steps at a time, tiles of pairs and small ones, tiles cut along K and joined in a cluster or by a launch of their own:
    sizes on both sides of the rules, the last ones with a K of hundreds of blocks."""
    u = normal(shape, gen(shape[0]), 1e-2)
    ref.close(lib.orthogonalize(u, bits=bits), ref.orthogonal(u), bits)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape,n", [((256, 64), 5), ((130, 260), 64), ((600, 256), 20), ((256, 256), 65), ((1024, 512), 6)], ids=str)
def test_batches(lib, shape, n, dtype):  # noqa: F811
    us = [normal(shape, gen(i), 1e-3 * (i + 1), dtype) for i in range(n)]
    for u, o in zip(us, lib.orthogonalize(us)):
        ref.close(o, ref.orthogonal(u), 32 if dtype == F32 else 16)


@pytest.mark.parametrize("shape", [(200, 96), (90, 3001)], ids=str)
@pytest.mark.parametrize("size", [2.0 ** -51.5, 2.0 ** 61])
def test_squares_near_the_ends_of_32_bits(lib, size, shape):  # noqa: F811
    """Eight squares are summed in 32 bits where they fit: sizes at which some eights of a matrix do and some do not."""
    u = (torch.randn(shape, generator=gen(3), device=DEV, dtype=torch.float64) * size).float()
    u[1::2, 8:24] = 0
    ref.close(lib.orthogonalize(u, eps=0.0), ref.orthogonal(u, eps=0.0), 32)


def test_many_of_low_rank(lib):  # noqa: F811
    """As many small matrices as are worth taking steps together."""
    for shape, rank in (((145, 2449), 30), ((164, 1311), 50), ((338, 131), 40), ((300, 1200), 60)):
        us = [normal((shape[0], rank), gen(2 * i)) @ normal((rank, shape[1]), gen(2 * i + 1)) for i in range(33)]
        for u, o in zip(us, lib.orthogonalize(us, bits=16)):
            ref.close(o, ref.orthogonal(u), 16)


def test_of_few_singular_values(lib):  # noqa: F811
    """Roundings of a few values do not average out: matrices as small as these take two terms whatever is asked for."""
    for i, shape in enumerate([(1, 1), (1, 1), (2, 6), (2, 1), (6, 3), (5, 2), (13, 2), (2, 9), (2, 3), (1, 700), (7, 7), (5, 5000)] * 20):
        u = normal(shape, gen(i))
        ref.close(lib.orthogonalize(u, bits=16), ref.orthogonal(u), 32)
        b = u.bfloat16()
        ref.close(lib.orthogonalize(b), ref.orthogonal(b), 32)


@pytest.mark.parametrize("steps", [5, 6])
@pytest.mark.parametrize("rank", [1, 2, 5])
@pytest.mark.parametrize("shape", [(4, 19), (7, 109), (145, 9), (2, 38), (21, 8), (300, 96), (1024, 256)], ids=str)
def test_of_low_rank(lib, shape, rank, steps):  # noqa: F811
    """What is not in the update's range stays small next to what is, in one matrix and in lists of them."""
    us = [normal((shape[0], rank), gen(8 * i)) @ normal((rank, shape[1]), gen(8 * i + 1)) for i in range(12 if shape[1] == 256 else 1)]
    for u, o in zip(us, lib.orthogonalize(us, bits=16, steps=steps)):
        ref.close(o, ref.orthogonal(u, steps=steps), 16, steps)


def test_two_streams_at_once(lib):  # noqa: F811
    """Calls that overlap have nothing in common but the status word."""
    sides = [torch.cuda.Stream() for _ in range(2)]
    us = [normal((1500, 700), gen(1)), normal((2000, 1500), gen(2), dtype=BF16)]
    want = [lib.orthogonalize(u) for u in us]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(6):
        for side, u, out in zip(sides, us, got):
            out.append(lib.orthogonalize(u, stream=side))
    torch.cuda.synchronize()
    for w, outs in zip(want, got):
        assert all(torch.equal(w, o) for o in outs)


def test_two_graphs_replayed_in_turn(lib):  # noqa: F811
    us = [normal((300, 500), gen(1)), normal((700, 600), gen(2))]
    want = [lib.orthogonalize(u) for u in us]
    graphs, outs = [torch.cuda.CUDAGraph() for _ in us], []
    for graph, u in zip(graphs, us):
        with torch.cuda.graph(graph):
            outs.append(lib.orthogonalize(u))
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(w, o) for w, o in zip(want, outs))


def test_a_model_of_many_shapes(lib):  # noqa: F811
    """More matrices than a launch takes, of several shapes and kinds, some empty: every one is stepped as its formula says."""
    g = gen(21)
    kinds = [("f32", (64, 48)), ("bf16", (64, 48)), ("master", (64, 48)), ("f32", (30, 90)), ("bf16", (257, 129)), ("master", (0, 48))]
    ts = [tensors(kinds[i % 6][1], kinds[i % 6][0], g) for i in range(210)]
    before = [copy(t) for t in ts]
    lists = [list(x) for x in zip(*ts)]
    lib.muon_step(lists[0], lists[1], lists[2], masters=lists[3], scale=0.7, **STEP)
    for i, (a, b) in enumerate(zip(before, ts)):
        if b[0].numel():
            check_step(a, b, STEP, 0.7, 16 if kinds[i % 6][0] == "bf16" else 32)


def test_serving_after_a_step_in_one_stream(lib):  # noqa: F811
    """An inference call may start reading weights before the work queued ahead of it has finished; a step holds it back."""
    D, H = 512, 2048
    g = gen(4)
    W = [normal((H, D), g, D ** -0.5, BF16) for _ in range(3)]
    grads = [normal((H, D), g, 1e-3, BF16) for _ in range(3)]
    served = lib.SparseFFN(D, H, BF16, device=DEV)
    x, bias = normal((D,), g, dtype=BF16), torch.full((H,), -0.5, device=DEV)
    start = [w.clone() for w in W]
    for wait in (True, False):
        for w, s in zip(W, start):
            w.copy_(s)
        states = [lib.muon_state(w) for w in W]
        torch.cuda.synchronize()
        for _ in range(3):
            lib.muon_step(W, grads, states, lr=0.05)
            if wait:
                torch.cuda.synchronize()
            y = served.sparse_ffn_forward(x, {"W_g": W[0]}, bias, W[1], W[2], "relu").clone()
        torch.cuda.synchronize()
        if wait:
            want = y
    assert torch.equal(y, want)


def test_a_step_before_a_forward_and_backward_pass(lib):  # noqa: F811
    """A training step's calls one after another without a synchronisation, twice, give the same bits."""
    def run():
        g = gen(7)
        W = [normal((300, 128), g, 0.1, BF16) for _ in range(3)]
        gain, states = torch.ones(128, device=DEV), None
        x = normal((200, 128), g, dtype=BF16)
        for _ in range(3):
            h, n, stats = lib.block_norm_forward(None, x, None, gain)
            y, z, u = lib.gated_ffn_forward(n, W[0], None, W[1], W[2], "silu")
            h2, n2, stats2 = lib.block_norm_forward(y, h, gain, gain)
            back = lib.block_norm_backward(h2, n2, y, h2, stats2, gain, gain)
            f = lib.gated_ffn_backward(back["dy"], n, z, u, W[0], W[1], W[2], "silu")
            grads = [f["dW_g"], f["dW_up"], f["dW_down"]]
            states = states or [lib.muon_state(w) for w in W]
            lib.muon_step(W, grads, states, lr=0.02, grad_norm=lib.grad_norm(grads), max_norm=1.0)
        return W + [s["m"] for s in states]

    assert all(torch.equal(a, b) for a, b in zip(run(), run()))


def test_offsets_beyond_32_bits(lib):  # noqa: F811
    """Rows so far apart that the last one starts beyond 2^32 elements."""
    R, C, ld = 3, 40, (1 << 31) - 64
    room = torch.zeros((R - 1) * ld + C, dtype=BF16, device=DEV)
    far = room.as_strided((R, C), (ld, 1))
    u = normal((R, C), gen(1), dtype=BF16)
    far.copy_(u)
    want = lib.orthogonalize(u)
    assert torch.equal(lib.orthogonalize(far), want)
    lib.orthogonalize(u, out=far)
    assert torch.equal(far, want)
