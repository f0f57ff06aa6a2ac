"""What the training calls keep between calls, when a call is captured into a CUDA graph.  Run with `-m gpu` on a B200."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture()
def lib(monkeypatch):
    import paper_2609_31975_b200 as m
    m.load_library()
    monkeypatch.setattr(m.training, "_kept", {})      # as in a process that has made no call yet
    yield m
    for knob, value in (("wait_cycles", 0), ("drop_stage", -1)):
        m.test_set_knob(knob, value)
    m.training_status(DEV, reset=True)


def test_a_wait_that_runs_out_in_a_replay_reaches_the_status(lib):
    """The first call of a process is a captured one; a copy that never comes, and a budget of a millisecond."""
    x, W = torch.ones(300, 256, device=DEV, dtype=torch.bfloat16), torch.ones(512, 256, device=DEV, dtype=torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    lib.test_set_knob("wait_cycles", 2_000_000)
    lib.test_set_knob("drop_stage", 1)
    with torch.cuda.graph(graph):
        lib.gated_ffn_forward(x, W, None, W, W)
    lib.test_set_knob("wait_cycles", 0)
    lib.test_set_knob("drop_stage", -1)
    assert lib.training_status(DEV) == 0
    graph.replay()
    assert lib.training_status(DEV) == 5
    lib.gated_ffn_forward(x, W, None, W, W)
    assert lib.training_status(DEV, reset=True) == 5 and lib.training_status(DEV) == 0
    graph.replay()
    assert lib.training_status(DEV, reset=True) == 5


def test_first_calls_in_a_capture(lib):
    """Every kind of call, none made before: the captured work computes what the calls compute by themselves."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x, dy = (torch.randn(70, 64, generator=g, device=DEV) for _ in range(2))
    W = [torch.randn(90, 64, generator=g, device=DEV) for _ in range(3)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, z, u = lib.gated_ffn_forward(x, W[0], None, W[1], W[2])
        grads = lib.gated_ffn_backward(dy, x, z, u, *W)
        norm = lib.grad_norm(list(grads.values()))
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    y1, z1, u1 = lib.gated_ffn_forward(x, W[0], None, W[1], W[2])
    more = lib.gated_ffn_backward(dy, x, z1, u1, *W)
    assert torch.equal(y, y1) and all(torch.equal(grads[k], more[k]) for k in more)
    assert torch.equal(norm, lib.grad_norm(list(more.values())))


def test_norms_captured_on_the_stream_of_earlier_norms(lib):
    """The graph's workspace is not the stream's: what the stream's holds does not reach a replay, and replays beside calls on the
    stream, and beside each other, leave each other's sums alone."""
    side = torch.cuda.Stream()
    tensors = [torch.full((1 << 20,), 0.5 + 0.25 * i, device=DEV) for i in range(3)]
    want = [lib.grad_norm([t]).item() for t in tensors]
    torch.cuda.synchronize()
    lib.grad_norm([tensors[0]], stream=side)                                    # warm-up, on the stream that is captured then
    graphs, norms = [], []
    for t in tensors[:2]:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            norms.append(lib.grad_norm([t]))
        graphs.append(graph)
    torch.cuda.synchronize()
    kept = lib.training._kept[0, side.cuda_stream, "norm"]
    before = kept.clone()
    kept.fill_(255)                                                             # a counter that no call would get past
    for n, graph in zip(norms, graphs):
        n.zero_()
        graph.replay()
    torch.cuda.synchronize()
    assert [n.item() for n in norms] == want[:2]
    kept.copy_(before)
    torch.cuda.synchronize()
    others = [torch.cuda.Stream() for _ in graphs]
    for _ in range(200):
        for n, graph, stream in zip(norms, graphs, others):
            with torch.cuda.stream(stream):
                n.zero_()
                graph.replay()
        third = lib.grad_norm([tensors[2]], stream=side)
        torch.cuda.synchronize()
        assert [n.item() for n in norms] == want[:2] and third.item() == want[2]
