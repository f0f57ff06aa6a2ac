"""CPU-side checks of the training calls: what they refuse before anything reaches a device, and the workspace they ask for."""
import ctypes

import pytest
import torch

import training_reference as ref

vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def lib():
    from paper_2609_31975_b200 import build

    build.build()
    import paper_2609_31975_b200 as m
    return m.load_library()


class Call(ctypes.Structure):
    _fields_ = [("T", ctypes.c_int32), ("D", ctypes.c_int32), ("H", ctypes.c_int32), ("dtype", ctypes.c_int32), ("act", ctypes.c_int32),
                ("act_up", ctypes.c_int32), ("x", vp), ("ld_x", ctypes.c_int64), ("W_g", vp), ("W_up", vp), ("W_down", vp), ("b_g", vp),
                ("z", vp), ("u", vp), ("ld_hidden", ctypes.c_int64), ("workspace", vp), ("workspace_bytes", ctypes.c_size_t), ("status", vp)]


class Grads(ctypes.Structure):
    _fields_ = [("dx", vp), ("ld_dx", ctypes.c_int64), ("dW_g", vp), ("dW_up", vp), ("dW_down", vp), ("db_g", vp)]


class Tensor(ctypes.Structure):
    _fields_ = [("data", vp), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class Step(ctypes.Structure):
    _fields_ = [("p", vp), ("g", vp), ("master", vp), ("m", vp), ("v", vp), ("m_scale", vp), ("v_scale", vp), ("n", ctypes.c_int64),
                ("p_dtype", ctypes.c_int32), ("g_dtype", ctypes.c_int32), ("state_bits", ctypes.c_int32), ("lr", ctypes.c_double),
                ("weight_decay", ctypes.c_double)]


class Config(ctypes.Structure):
    _fields_ = [("beta1", ctypes.c_double), ("beta2", ctypes.c_double), ("eps", ctypes.c_double), ("step", ctypes.c_int64),
                ("grad_norm", vp), ("max_norm", ctypes.c_double)]


A = 1 << 20  # an address on 16 and 256 bytes that nothing reads: every call below is refused before


def good(**over):
    c = Call(16, 64, 40, 1, 0, 3, A, 64, A, A, A, None, A, A, 40, A, 1 << 40, A)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def test_workspace(lib):
    need = ctypes.c_size_t(0)
    ask = lambda *a: lib.sffn_train_workspace_bytes(*a, ctypes.byref(need))  # noqa: E731
    assert ask(8192, 4096, 14336, 1, 0) == 0 and need.value >= 8192 * 14336 * 2
    forward = need.value
    assert ask(8192, 4096, 14336, 1, 1) == 0 and need.value >= forward + 2 * 8192 * 14336 * 2
    assert ask(500, 3840, 14230, 0, 1) == 0 and need.value >= 3 * 3840 * 14230 * 6   # the weights' three terms
    assert ask(0, 64, 40, 1, 0) == 0 and need.value >= 256
    assert ask(-1, 64, 40, 1, 0) == 1 and ask(1, 0, 40, 1, 0) == 1 and ask(1, 64, 0, 1, 0) == 1 and ask(1, 64, 40, 2, 0) == 1
    assert ask(1, 60, 40, 1, 0) == 2 and ask(1, 66, 40, 0, 0) == 2 and ask(1, 60, 40, 0, 0) == 0
    assert ask(1 << 23, 64, 40, 1, 0) == 2
    assert lib.sffn_train_workspace_bytes(1, 64, 40, 1, 0, None) == 1


@pytest.mark.parametrize("over,code", [
    (dict(T=-1), 1), (dict(D=0), 1), (dict(H=0), 1), (dict(dtype=3), 1), (dict(act=5), 1), (dict(act=-1), 1), (dict(act_up=7), 1),
    (dict(x=None), 1), (dict(W_g=None), 1), (dict(W_down=None), 1), (dict(status=None), 1), (dict(ld_x=56), 1), (dict(ld_hidden=32), 1),
    (dict(z=None), 1), (dict(u=None), 1),
    (dict(D=60, ld_x=64), 2), (dict(x=A + 8), 2), (dict(ld_x=68), 2), (dict(W_up=A + 2), 2), (dict(ld_hidden=44), 2), (dict(u=A + 4), 2), (dict(b_g=A + 2), 2),
    (dict(workspace=None), 3), (dict(workspace=A + 16), 3), (dict(workspace_bytes=64), 3)])
def test_refused_calls(lib, over, code):
    c, g = good(**over), Grads(A, 64, A, A, A, A)
    assert lib.gated_ffn_forward(ctypes.byref(c), vp(A), ctypes.c_int64(64), None) == code
    assert lib.gated_ffn_backward(ctypes.byref(c), vp(A), ctypes.c_int64(64), ctypes.byref(g), None) == code


def test_refused_outputs(lib):
    c = good()
    i64 = ctypes.c_int64
    assert lib.gated_ffn_forward(None, vp(A), i64(64), None) == 1
    assert lib.gated_ffn_forward(ctypes.byref(c), None, i64(64), None) == 1
    assert lib.gated_ffn_forward(ctypes.byref(c), vp(A), i64(32), None) == 1
    assert lib.gated_ffn_forward(ctypes.byref(c), vp(A + 4), i64(64), None) == 2
    assert lib.gated_ffn_backward(ctypes.byref(c), vp(A), i64(64), None, None) == 1
    for g, code in ((Grads(A, 60, A, A, A, A), 1), (Grads(A + 2, 64, A, A, A, A), 2), (Grads(A, 64, A + 2, A, A, A), 2), (Grads(A, 64, A, A, A, A + 1), 2)):
        assert lib.gated_ffn_backward(ctypes.byref(c), vp(A), i64(64), ctypes.byref(g), None) == code
    assert lib.gated_ffn_backward(ctypes.byref(c), None, i64(64), ctypes.byref(Grads(A, 64)), None) == 1
    assert lib.gated_ffn_backward(ctypes.byref(c), vp(A), i64(64), ctypes.byref(Grads()), None) == 0     # nothing is wanted
    none = good(T=0, x=None, z=None, u=None)
    assert lib.gated_ffn_forward(ctypes.byref(none), None, i64(0), None) == 0                           # no tokens, nothing to do


def test_refused_norms_and_steps(lib):
    t = (Tensor * 1)(Tensor(A, 8, 1))
    norm = lambda t, n, out=A, ws=A, size=16384: lib.sffn_grad_norm(t, n, vp(out), vp(ws), ctypes.c_size_t(size), None)  # noqa: E731
    assert norm(t, -1) == 1 and norm(None, 1) == 1 and norm(t, 1, out=None) == 1 and norm(t, 1, ws=None) == 3 and norm(t, 1, size=100) == 3
    assert norm(t, 1, out=A + 2) == 2
    for bad, code in ((Tensor(None, 8, 1), 1), (Tensor(A, -8, 1), 1), (Tensor(A, 8, 2), 1), (Tensor(A + 1, 8, 1), 2), (Tensor(A, 1 << 40, 1), 2)):
        assert norm((Tensor * 1)(bad), 1) == code
    fine = dict(p=A, g=A, m=A, v=A, m_scale=A, v_scale=A, n=8, p_dtype=1, g_dtype=1, state_bits=8, lr=1e-3, weight_decay=0.1)
    conf = dict(beta1=0.9, beta2=0.99, eps=1e-8, step=1)

    def step(conf_over=None, **over):
        a = (Step * 1)(Step(**dict(fine, **over)))
        return lib.sffn_adamw_step(a, 1, ctypes.byref(Config(**dict(conf, **(conf_over or {})))), None)

    for over, code in ((dict(p=None), 1), (dict(g=None), 1), (dict(m=None), 1), (dict(v_scale=None), 1), (dict(n=-1), 1), (dict(state_bits=16), 1),
                       (dict(p_dtype=2), 1), (dict(g_dtype=9), 1), (dict(p_dtype=0, master=A), 1), (dict(lr=float("inf")), 1), (dict(p=A + 1), 2),
                       (dict(master=A + 2), 2), (dict(m_scale=A + 2), 2), (dict(n=1 << 40), 2), (dict(state_bits=32, m=A + 2), 2)):
        assert step(**over) == code, over
    for over in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.5), dict(eps=-1.0), dict(eps=float("inf")), dict(grad_norm=A, max_norm=0.0), dict(beta1=float("nan"))):
        assert step(over) == 1, over
    assert lib.sffn_adamw_step(None, 1, ctypes.byref(Config(**conf)), None) == 1
    assert lib.sffn_adamw_step((Step * 1)(Step(**fine)), 1, None, None) == 1
    a = (Step * 1)(Step(**dict(fine, state_bits=32)))
    assert lib.sffn_adamw_state_values(a, 1, None, None, None) == 1


def test_tensors_that_are_not_on_a_device_are_refused(lib):
    import paper_2609_31975_b200 as m
    w = torch.zeros(8, 8)
    for f in (lambda: m.gated_ffn_forward(w, w, None, w, w), lambda: m.gated_ffn_backward(w, w, w, w, w, w, w), lambda: m.grad_norm([w]),
              lambda: m.adamw_step([w], [w], [m.adamw_state(w)], 1, lr=1e-3), lambda: m.adamw_state_values([m.adamw_state(w, 8)])):
        with pytest.raises(TypeError, match="CUDA"):
            f()


def test_plain_forms_agree_with_torch():
    """The reference of the GPU tests against torch's own differentiation, in 64 bits."""
    g = torch.Generator().manual_seed(3)
    T, D, H = 7, 12, 9
    x, W = torch.randn(T, D, generator=g).double(), [torch.randn(H, D, generator=g).double() for _ in range(3)]
    b, dy = torch.randn(H, generator=g).double(), torch.randn(T, D, generator=g).double()
    torch_act = {"relu": torch.relu, "sqrelu": lambda t: torch.relu(t) ** 2, "rsplus": lambda t: torch.nn.functional.silu(torch.relu(t)) * (t > 0),
                 "silu": torch.nn.functional.silu, None: lambda t: t}
    for a in ("relu", "sqrelu", "rsplus", "silu", None):
        for a_up in (None, "relu", "silu"):
            leaves = [t.clone().requires_grad_() for t in (x, W[0], b, W[1], W[2])]
            z, u = leaves[0] @ leaves[1].T + leaves[2], leaves[0] @ leaves[3].T
            y = (torch_act[a](z) * torch_act[a_up](u)) @ leaves[4]
            grads = torch.autograd.grad(y, leaves, dy)
            f = ref.forward(x, W[0], b, W[1], W[2], a, a_up)
            assert torch.allclose(f["y"], y, atol=1e-12)
            got = ref.backward(dy, x, f["z"], f["u"], *W, a, a_up)
            for k, want in zip(("dx", "dW_g", "db_g", "dW_up", "dW_down"), grads):
                assert torch.allclose(got[k], want, atol=1e-11), (a, a_up, k)
