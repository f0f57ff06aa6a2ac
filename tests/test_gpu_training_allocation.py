"""What a call makes and returns is made as torch's own operations make it: dispatch modes see it, and under deterministic algorithms memory that
nothing has written yet is filled.  Run with `-m gpu` on a B200."""
import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    return m


class Made(TorchDispatchMode):
    def __init__(self):
        super().__init__()
        self.shapes = []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if func is torch.ops.aten.empty.memory_format:
            self.shapes.append(tuple(out.shape))
        return out


def weights(D, H):
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    return [torch.randn(H, D, generator=g, device=DEV) * D ** -0.5 for _ in range(3)]


@pytest.mark.parametrize("inference", [False, True])
def test_dispatch_modes_see_what_is_made(lib, inference):
    T, D, H = 5, 64, 44
    W, x, gain = weights(D, H), torch.ones(T, D, device=DEV), torch.ones(D, device=DEV)
    calls = {"forward": (lambda: lib.gated_ffn_forward(x, W[0], None, W[1], W[2]), (T, D)), "norm": (lambda: lib.grad_norm([x]), ()),
             "block": (lambda: lib.block_norm_forward(x, x, gain, gain), (2, T)), "orthogonalize": (lambda: lib.orthogonalize(W[0]), (H, D))}
    with torch.inference_mode(inference):
        for name, (call, shape) in calls.items():
            call()
            with Made() as mode:
                call()
            assert shape in mode.shapes, (name, mode.shapes)


def test_deterministic_algorithms_fill(lib):
    T, D, H = 5, 64, 44  # rows of z and u end before their stride
    W, x = weights(D, H), torch.ones(T, D, device=DEV)
    want = lib.gated_ffn_forward(x, W[0], None, W[1], W[2])
    torch.full((1 << 20,), 7.0, device=DEV)
    assert torch.utils.deterministic.fill_uninitialized_memory
    torch.use_deterministic_algorithms(True)
    try:
        y, z, u = lib.gated_ffn_forward(x, W[0], None, W[1], W[2])
        dW = lib.gated_ffn_backward(x, x, z, u, *W)
    finally:
        torch.use_deterministic_algorithms(False)
    assert all(torch.equal(a, b) for a, b in zip((y, z, u), want))
    for t in (z, u):
        past = torch.as_strided(t, (T - 1, t.stride(0)), t.stride())[:, H:]
        assert past.numel() and past.isnan().all()
    again = lib.gated_ffn_backward(x, x, want[1], want[2], *W)
    assert all(torch.equal(dW[k], again[k]) for k in again)
