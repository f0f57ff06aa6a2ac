"""CPU-side checks of the norms around a block: what they refuse before anything reaches a device."""
import ctypes

import pytest

vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float


@pytest.fixture(scope="module")
def lib():
    from paper_2609_31975_b200 import build

    build.build()
    import paper_2609_31975_b200 as m
    return m.load_library()


class Call(ctypes.Structure):
    _fields_ = [("T", i32), ("D", i32), ("y_dtype", i32), ("h_dtype", i32), ("n_dtype", i32), ("gate_kind", i32), ("y", vp), ("ld_y", i64), ("resid", vp),
                ("ld_resid", i64), ("post_gain", vp), ("pre_gain", vp), ("gate", vp), ("ld_gate", i64), ("scale", f32), ("eps", f32), ("h", vp), ("ld_h", i64),
                ("n", vp), ("ld_n", i64), ("stats", vp)]


class Grads(ctypes.Structure):
    _fields_ = [("dh", vp), ("ld_dh", i64), ("dn", vp), ("ld_dn", i64), ("dy", vp), ("ld_dy", i64), ("dresid", vp), ("ld_dresid", i64), ("dpost_gain", vp),
                ("dpre_gain", vp), ("dgate", vp), ("ld_dgate", i64), ("workspace", vp), ("workspace_bytes", ctypes.c_size_t)]


A, STEP = 1 << 30, 1 << 24  # addresses on 256 bytes that nothing reads: every call below is refused before


def at(n):
    return A + n * STEP


def call(**over):
    c = Call(16, 64, 1, 1, 1, 3, at(0), 64, at(1), 64, at(2), at(3), at(4), 64, 1.0, 1e-6, at(5), 64, at(6), 64, at(7))
    for k, v in over.items():
        setattr(c, k, v)
    return c


def grads(**over):
    g = Grads(at(8), 64, at(9), 64, at(10), 64, at(11), 64, at(12), at(13), at(14), 64, at(15), 1 << 30)
    for k, v in over.items():
        setattr(g, k, v)
    return g


INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
EITHER = [(dict(T=-1), 1), (dict(D=0), 1), (dict(y_dtype=2), 1), (dict(h_dtype=-1), 1), (dict(n_dtype=7), 1), (dict(gate_kind=4), 1), (dict(gate_kind=-1), 1),
          (dict(scale=float("nan")), 1), (dict(eps=-1e-6), 1), (dict(eps=float("inf")), 1), (dict(eps=float("nan")), 1), (dict(gate=None), 1), (dict(ld_y=56), 1),
          (dict(ld_gate=8), 1), (dict(y=None), 1),
          (dict(D=60), 2), (dict(D=62, y_dtype=0, h_dtype=0, n_dtype=0), 2), (dict(D=32776, ld_y=32776), 2), (dict(y=at(0) + 8), 2), (dict(ld_y=68), 2),
          (dict(post_gain=at(2) + 4), 2), (dict(pre_gain=at(3) + 8), 2), (dict(gate=at(4) + 4), 2), (dict(gate_kind=1, gate=at(4) + 4), 2),
          (dict(gate_kind=2, gate=at(4) + 2), 2), (dict(stats=at(7) + 2), 2), (dict(ld_h=1 << 40), 2)]


@pytest.mark.parametrize("over,code", EITHER)
def test_refused_by_both(lib, over, code):
    assert lib.sffn_block_norm_forward(ctypes.byref(call(**over)), None) == code
    assert lib.sffn_block_norm_backward(ctypes.byref(call(**over)), ctypes.byref(grads()), None) == code


@pytest.mark.parametrize("over,code", [
    (dict(h=None), 1), (dict(n=None), 1), (dict(ld_n=60), 1), (dict(n=at(6) + 2), 2), (dict(resid=at(1) + 4), 2), (dict(h=at(0)), 1), (dict(n=at(1)), 1),
    (dict(n=at(5) + 16), 1), (dict(h=at(1) + 16), 1), (dict(h=at(1), ld_h=72), 1), (dict(stats=at(6)), 1), (dict(stats=at(1) + 32), 1), (dict(h=at(4)), 1), (dict(n=at(3)), 1),
    (dict(y=None, gate_kind=0, post_gain=None, resid=None), 1), (dict(y=None, gate_kind=0, post_gain=None, pre_gain=None), 1)])
def test_refused_forward(lib, over, code):
    assert lib.sffn_block_norm_forward(ctypes.byref(call(**over)), None) == code


@pytest.mark.parametrize("over,more,code", [
    ({}, dict(dh=None, dn=None), 1), (dict(stats=None), {}, 1), (dict(h=None), {}, 1), (dict(pre_gain=None), {}, 1), (dict(post_gain=None), {}, 1),
    (dict(gate_kind=0), {}, 1), ({}, dict(ld_dy=8), 1), ({}, dict(dy=at(0)), 1), ({}, dict(dy=at(8)), 1), ({}, dict(dresid=at(9)), 1), ({}, dict(dresid=at(8) + 16), 1),
    ({}, dict(dresid=at(8), ld_dresid=72), 1), ({}, dict(dpre_gain=at(12)), 1), ({}, dict(dgate=at(4)), 1), ({}, dict(dy=at(15) + 256), 1), ({}, dict(dy=at(5)), 1),
    ({}, dict(dy=at(10) + 2), 2), ({}, dict(dpost_gain=at(12) + 4), 2), ({}, dict(dgate=at(14) + 2), 2), ({}, dict(ld_dh=66), 2),
    ({}, dict(workspace=None), 3), ({}, dict(workspace=at(15) + 4), 3), ({}, dict(workspace_bytes=1000), 3)])
def test_refused_backward(lib, over, more, code):
    assert lib.sffn_block_norm_backward(ctypes.byref(call(**over)), ctypes.byref(grads(**more)), None) == code


def test_nothing_to_do(lib):
    """No tokens (and then no addresses), or no gradient asked for: fine, and nothing reaches a device."""
    c = call(T=0, y=None, resid=None, h=None, n=None, gate=None, stats=None)
    assert lib.sffn_block_norm_forward(ctypes.byref(c), None) == 0
    nothing = dict(dy=None, dresid=None, dpost_gain=None, dpre_gain=None, dgate=None)
    assert lib.sffn_block_norm_backward(ctypes.byref(c), ctypes.byref(grads(dh=None, dn=None, **nothing)), None) == 0
    assert lib.sffn_block_norm_backward(ctypes.byref(call()), ctypes.byref(grads(**nothing)), None) == 0
    assert lib.sffn_block_norm_forward(None, None) == 1 and lib.sffn_block_norm_backward(None, None, None) == 1
    assert lib.sffn_block_norm_backward(ctypes.byref(call()), None, None) == 1


def test_workspace(lib):
    need = ctypes.c_size_t(0)
    ask = lambda D: lib.sffn_block_norm_workspace_bytes(D, ctypes.byref(need))  # noqa: E731
    assert ask(4096) == 0 and need.value >= 2 * 148 * 2 * 4096 * 4
    assert ask(8) == 0 and ask(32768) == 0 and ask(32772) == 2 and ask(6) == 2 and ask(0) == 1
    assert lib.sffn_block_norm_workspace_bytes(64, None) == 1
