"""The training calls when a wait inside a kernel runs out: a copy that never comes, with the wait budget cut to a millisecond.
The kernels come back by themselves, leave SFFN_ERR_TIMEOUT in the status word and give back shared and tensor memory, and the
next call computes as before."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SHORT = 2_000_000        # cycles: about a millisecond


@pytest.fixture()
def lib():
    import paper_2609_31975_b200 as m
    m.load_library()
    m.training_status(DEV, reset=True)
    yield m
    for knob, value in (("wait_cycles", 0), ("drop_stage", -1)):
        m.test_set_knob(knob, value)
    m.training_status(DEV, reset=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=["bf16", "f32"])
def test_a_copy_that_never_comes(lib, dtype):
    T, D, H = 520, 520, 1000      # on the tensor cores in either type
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV).to(dtype)  # noqa: E731
    x, dy, W, b_g = rnd(T, D), rnd(T, D), [rnd(H, D) for _ in range(3)], torch.zeros(H, device=DEV)
    y, z, u = lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2])
    grads = lib.gated_ffn_backward(dy, x, z, u, *W)
    assert lib.training_status(DEV) == 0
    for stage in (0, 1):
        lib.test_set_knob("wait_cycles", SHORT)
        lib.test_set_knob("drop_stage", stage)
        lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2])
        assert lib.training_status(DEV) == 5                 # SFFN_ERR_TIMEOUT, and it stays
        assert lib.training_status(DEV, reset=True) == 5 and lib.training_status(DEV) == 0
        lib.gated_ffn_backward(dy, x, z, u, *W)
        assert lib.training_status(DEV, reset=True) == 5
        lib.test_set_knob("wait_cycles", 0)
        lib.test_set_knob("drop_stage", -1)
        again = lib.gated_ffn_forward(x, W[0], b_g, W[1], W[2])
        more = lib.gated_ffn_backward(dy, x, z, u, *W)
        assert lib.training_status(DEV) == 0
        assert all(torch.equal(p, q) for p, q in zip((y, z, u), again)) and all(torch.equal(grads[k], more[k]) for k in grads)


def test_synchronising_mode_names_the_call(lib, monkeypatch):
    x, W = torch.ones(300, 256, device=DEV, dtype=torch.bfloat16), torch.ones(512, 256, device=DEV, dtype=torch.bfloat16)
    monkeypatch.setenv("SFFN_SYNC_CHECK", "1")
    lib.gated_ffn_forward(x, W, None, W, W)
    lib.test_set_knob("wait_cycles", SHORT)
    lib.test_set_knob("drop_stage", 1)
    with pytest.raises(RuntimeError, match="gated_ffn_forward: device status 5"):
        lib.gated_ffn_forward(x, W, None, W, W)
