"""What the training calls write into a caller's tensors is seen by torch's version counters.  Run with `-m gpu` on a B200."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    return m


def make(T=24, D=64, H=40, dtype=torch.bfloat16):
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)  # noqa: E731
    return rnd(T, D), [rnd(H, D) for _ in range(3)], torch.zeros(H, device=DEV), rnd(T, D)


@pytest.mark.parametrize("bits", [8, 32])
def test_a_backward_pass_after_a_step_raises(lib, bits):
    x, (W_g, W_up, W_down), b_g, _ = make()
    for w in (W_g, W_up, W_down):
        w.requires_grad_()
    y = lib.GatedFFNFunction.apply(x, W_g, b_g, W_up, W_down, "silu")
    grad = torch.zeros_like(W_up)
    lib.adamw_step([W_up], [grad], [lib.adamw_state(W_up, bits)], 1, lr=1e-3)
    with pytest.raises(RuntimeError, match="inplace"):
        y.sum().backward()
    y = lib.GatedFFNFunction.apply(x, W_g, b_g, W_up, W_down, "silu")     # and the next pass is a pass like any other
    y.sum().backward()
    assert W_up.grad is not None


def test_every_tensor_that_a_call_writes_counts(lib):
    x, W, b_g, dy = make()
    rows = lambda n, dtype=torch.bfloat16: torch.empty(24, n, dtype=dtype, device=DEV)  # noqa: E731

    def counted(tensors, call, others=()):
        before = [t._version for t in (*tensors, *others)]
        call()
        after = [t._version for t in (*tensors, *others)]
        assert all(a > b for a, b in zip(after[:len(tensors)], before))
        assert after[len(tensors):] == before[len(tensors):]

    y, z, u = rows(64), rows(40), rows(40)
    read = (x, *W, b_g, dy)
    counted([y, z, u], lambda: lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2], y=y, z=z, u=u), read)
    counted([y], lambda: lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2], save=False, y=y), (z, u))
    out = dict(dx=rows(64), dW_g=torch.empty_like(W[0]), db_g=torch.empty(40, device=DEV))
    counted(list(out.values()), lambda: lib.gated_ffn_backward(dy, x, z, u, *W, out=out), (z, u, *read))
    norm = torch.empty((), device=DEV)
    counted([norm], lambda: lib.grad_norm([dy], norm), (dy,))
    for bits in (8, 32):
        state, master, grad = lib.adamw_state(W[0], bits), W[0].float(), torch.ones_like(W[0])
        counted([W[0], master, *state.values()], lambda: lib.adamw_step([W[0]], [grad], [state], 1, lr=1e-3, masters=[master], grad_norm=norm), (grad, norm))
        if bits == 8:
            values = [dict(m=torch.empty(40, 64, device=DEV), v=torch.empty(40, 64, device=DEV))]
            counted(list(values[0].values()), lambda: lib.adamw_state_values([state], values), state.values())
    narrow = torch.empty(24, 66, dtype=torch.bfloat16, device=DEV)
    before = narrow._version
    with pytest.raises(lib.SFFNError):
        lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2], y=narrow[:, :64])
    assert narrow._version == before


def test_tensors_of_inference_mode_are_taken(lib):
    with torch.inference_mode():
        w = torch.ones(64, device=DEV)
        state = lib.adamw_state(w)
    lib.adamw_step([w], [torch.ones(64, device=DEV)], [state], 1, lr=0.5, weight_decay=0.0)
    assert torch.allclose(w, torch.full((64,), 0.5, device=DEV), atol=1e-6)
