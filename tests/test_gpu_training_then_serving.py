"""A step and the inference calls that follow it on the same stream, without a synchronisation between them: they compute with the new
weights.  Run with `-m gpu` on a B200."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    return m


@pytest.mark.parametrize("bits,master", [(32, False), (8, False), (8, True)])
@pytest.mark.parametrize("B", [1, 16])
def test_serving_right_after_a_step(lib, bits, master, B):
    D, H, rounds = 2048, 8192, 6
    g = torch.Generator(device=DEV)
    g.manual_seed(bits + B)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    start = [(rnd(H, D) * D ** -0.5).bfloat16() for _ in range(3)]
    grads = [[rnd(H, D).bfloat16() for _ in range(3)] for _ in range(rounds)]
    x, b_g = rnd(B, D).bfloat16(), rnd(H) - 1.0
    ffn = lib.SparseFFN(D, H, torch.bfloat16, B_max=B, device=DEV)

    def run(meet):
        W = [w.clone() for w in start]
        copies = [w.float() for w in W] if master else None
        states = [lib.adamw_state(w, bits) for w in W]
        torch.cuda.synchronize()
        out = []
        for step in range(rounds):
            lib.adamw_step(W, grads[step], states, step + 1, lr=2e-2, masters=copies)
            if meet:
                torch.cuda.synchronize()
            out.append(ffn.sparse_ffn_forward(x, {"W_g": W[0]}, b_g, W[1], W[2], "relu").clone())
            torch.cuda.synchronize()
        return out

    want = run(True)
    assert all(not torch.equal(a, b) for a, b in zip(want, want[1:]))          # a step changes the output
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(False), want))


@pytest.mark.parametrize("B", [1, 16])
def test_serving_right_after_a_step_in_a_graph(lib, B):
    D, H, rounds = 2048, 8192, 6
    g = torch.Generator(device=DEV)
    g.manual_seed(B)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    start, grads = [(rnd(H, D) * D ** -0.5).bfloat16() for _ in range(3)], [rnd(H, D).bfloat16() for _ in range(3)]
    x, b_g = rnd(B, D).bfloat16(), rnd(H) - 1.0
    ffn = lib.SparseFFN(D, H, torch.bfloat16, B_max=B, device=DEV)

    def pieces():
        W = [w.clone() for w in start]
        return W, [lib.adamw_state(w, 8) for w in W]

    W, states = pieces()
    want = []
    for _ in range(rounds):
        lib.adamw_step(W, grads, states, 1, lr=2e-2)
        torch.cuda.synchronize()
        want.append(ffn.sparse_ffn_forward(x, {"W_g": W[0]}, b_g, W[1], W[2], "relu").clone())
        torch.cuda.synchronize()
    W, states = pieces()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        lib.adamw_step(W, grads, states, 1, lr=2e-2)
        y = ffn.sparse_ffn_forward(x, {"W_g": W[0]}, b_g, W[1], W[2], "relu")
    got = []
    for _ in range(rounds):
        graph.replay()
        got.append(y.clone())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(not torch.equal(a, b) for a, b in zip(want, want[1:]))
