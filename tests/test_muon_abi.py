"""CPU-side checks of the orthogonalised update and the Muon step: what they refuse before anything reaches a device, and the workspace
they ask for."""
import ctypes

import pytest

vp, i32, i64, f64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_double


@pytest.fixture(scope="module")
def lib():
    from paper_2609_31975_b200 import build

    build.build()
    import paper_2609_31975_b200 as m
    return m.load_library()


class NewtonSchulz(ctypes.Structure):
    _fields_ = [("steps", i32), ("bits", i32), ("coefficients", ctypes.POINTER(f64)), ("eps", f64)]


class Orthogonal(ctypes.Structure):
    _fields_ = [("u", vp), ("ld_u", i64), ("o", vp), ("ld_o", i64), ("rows", i32), ("cols", i32), ("dtype", i32)]


class Tensor(ctypes.Structure):
    _fields_ = [("p", vp), ("g", vp), ("master", vp), ("m", vp), ("rows", i32), ("cols", i32), ("p_dtype", i32), ("g_dtype", i32), ("lr", f64),
                ("weight_decay", f64), ("scale", f64)]


class Config(ctypes.Structure):
    _fields_ = [("ns", NewtonSchulz), ("momentum", f64), ("nesterov", i32), ("grad_norm", vp), ("max_norm", f64)]


A, STEP, WS = 1 << 30, 1 << 24, 1 << 40  # addresses on 256 bytes that nothing reads: every call below is refused before


def at(n):
    return A + n * STEP


def ns(steps=5, bits=0, triples=None, eps=1e-7, **over):
    values = triples if triples is not None else [3.4445, -4.7750, 2.0315] * max(steps, 0)
    out = NewtonSchulz(steps, bits, (f64 * max(len(values), 1))(*values), eps)
    for k, v in over.items():
        setattr(out, k, v)
    return out


def orthogonal(**over):
    t = Orthogonal(at(0), 40, at(1), 40, 64, 40, 1)
    for k, v in over.items():
        setattr(t, k, v)
    return t


def tensor(base=0, **over):
    t = Tensor(at(base), at(base + 1), at(base + 2), at(base + 3), 64, 40, 1, 1, 0.02, 0.1, 1.0)
    for k, v in over.items():
        setattr(t, k, v)
    return t


def config(**over):
    c = Config(ns(), 0.95, 1, None, 0.0)
    for k, v in over.items():
        setattr(c, k, v)
    return c


def call_orthogonal(lib, ts, how=None, ws=WS, room=1 << 40, status=at(40)):
    array = (Orthogonal * max(len(ts), 1))(*ts)
    return lib.sffn_orthogonalize(array, len(ts), ctypes.byref(how or ns()), vp(ws), ctypes.c_size_t(room), vp(status), None)


def call_step(lib, ts, c=None, ws=WS, room=1 << 40, status=at(40)):
    array = (Tensor * max(len(ts), 1))(*ts)
    return lib.sffn_muon_step(array, len(ts), ctypes.byref(c or config()), vp(ws), ctypes.c_size_t(room), vp(status), None)


@pytest.mark.parametrize("how", [dict(steps=0), dict(steps=-1), dict(steps=33), dict(bits=8), dict(bits=-1), dict(eps=-1e-9), dict(eps=float("inf")), dict(eps=float("nan")),
                                 dict(coefficients=None), dict(steps=1, triples=[1.0, float("inf"), 0.0]), dict(steps=2, triples=[1e9, 0.0, 0.0] * 2),
                                 dict(steps=5, triples=[100.0, 100.0, 100.0] * 5)])
def test_refused_steps(lib, how):
    assert call_orthogonal(lib, [orthogonal()], ns(**how)) == 1
    assert call_step(lib, [tensor()], config(ns=ns(**how))) == 1
    need = ctypes.c_size_t(0)
    assert lib.sffn_orthogonalize_workspace_bytes(ctypes.byref(orthogonal()), 1, ctypes.byref(ns(**how)), ctypes.byref(need)) == 1


@pytest.mark.parametrize("over,code", [(dict(rows=-1), 1), (dict(cols=-1), 1), (dict(dtype=2), 1), (dict(u=None), 1), (dict(o=None), 1), (dict(ld_u=39), 1), (dict(ld_o=0), 1),
                                       (dict(rows=1 << 17, cols=1 << 17, ld_u=1 << 17, ld_o=1 << 17), 2), (dict(rows=1 << 23), 2), (dict(u=at(0) + 1), 2),
                                       (dict(dtype=0, o=at(1) + 2), 2), (dict(ld_u=1 << 41), 2), (dict(o=at(0) + 80), 0), (dict(o=WS + 1024), 1), (dict(o=at(40)), 1)])
def test_refused_updates(lib, over, code):
    if code:
        assert call_orthogonal(lib, [orthogonal(**over)]) == code
    else:  # an output over its own update: only another matrix's makes it wrong
        assert call_orthogonal(lib, [orthogonal(**over), orthogonal(u=at(2), o=at(0))]) == 1


def test_refused_lists(lib):
    assert lib.sffn_orthogonalize(None, 1, ctypes.byref(ns()), vp(WS), ctypes.c_size_t(1 << 40), vp(at(40)), None) == 1
    assert lib.sffn_orthogonalize(None, -1, ctypes.byref(ns()), vp(WS), ctypes.c_size_t(1 << 40), vp(at(40)), None) == 1
    one, two = orthogonal(), orthogonal(u=at(2), o=at(3))
    assert call_orthogonal(lib, [one, two], ws=None) == 3 and call_orthogonal(lib, [one, two], ws=WS + 16) == 3 and call_orthogonal(lib, [one, two], room=1000) == 3
    assert call_orthogonal(lib, [one, two], status=None) == 1 and call_orthogonal(lib, [one, two], status=at(40) + 2) == 2
    for bad in (dict(o=at(1)), dict(o=at(1) + 64 * 80 - 2), dict(o=at(0) + 2), dict(u=at(1)), dict(u=at(1) + 8, ld_u=72)):
        assert call_orthogonal(lib, [one, orthogonal(**{**dict(u=at(2), o=at(3)), **bad})]) == 1, bad
    # columns of one matrix do not meet; with one column too many they do
    left, right = (orthogonal(o=at(5) + 80 * i, ld_o=80) for i in (0, 1))
    right.u = at(2)
    wider = orthogonal(u=at(2), o=at(5) + 78, ld_o=80)
    assert call_orthogonal(lib, [left, wider]) == 1 and call_orthogonal(lib, [left, right], room=1000) == 3


@pytest.mark.parametrize("over,code", [(dict(rows=-1), 1), (dict(p_dtype=3), 1), (dict(g_dtype=-1), 1), (dict(p_dtype=0), 1), (dict(p=None), 1), (dict(g=None), 1), (dict(m=None), 1),
                                       (dict(lr=float("nan")), 1), (dict(weight_decay=float("inf")), 1), (dict(scale=float("nan")), 1), (dict(rows=1 << 23), 2),
                                       (dict(p=at(0) + 1), 2), (dict(g=at(1) + 1), 2), (dict(m=at(3) + 2), 2), (dict(master=at(2) + 2), 2),
                                       (dict(g=at(0)), 1), (dict(m=at(1)), 1), (dict(master=at(3) + 64), 1), (dict(p=WS + 512), 1), (dict(m=at(40)), 1)])
def test_refused_tensors(lib, over, code):
    assert call_step(lib, [tensor(**over)]) == code


def test_refused_configurations(lib):
    for over in (dict(momentum=1.0), dict(momentum=-0.1), dict(momentum=float("nan")), dict(grad_norm=at(30), max_norm=0.0), dict(grad_norm=at(30), max_norm=float("nan"))):
        assert call_step(lib, [tensor()], config(**over)) == 1
    assert call_step(lib, [tensor()], config(grad_norm=at(30) + 2, max_norm=1.0)) == 2
    assert call_step(lib, [tensor()], config(grad_norm=at(0), max_norm=1.0)) == 1            # the norm's word inside a parameter
    assert call_step(lib, [tensor(), tensor(base=3)]) == 1 and call_step(lib, [tensor(), tensor()]) == 1
    assert call_step(lib, [tensor(), tensor(base=4, g=at(1))], room=1000) == 3                   # one gradient for two: fine, but for the room
    assert call_step(lib, [tensor()], ws=None) == 3 and call_step(lib, [tensor()], status=None) == 1
    array = (Tensor * 1)(tensor())
    assert lib.sffn_muon_step(array, 1, None, vp(WS), ctypes.c_size_t(1 << 40), vp(at(40)), None) == 1


def test_workspace(lib):
    def ask(shapes, bits=0, dtype=1):
        need = ctypes.c_size_t(0)
        array = (Orthogonal * max(len(shapes), 1))(*[Orthogonal(None, 0, None, 0, r, c, dtype) for r, c in shapes])
        assert lib.sffn_orthogonalize_workspace_bytes(array, len(shapes), ctypes.byref(ns(bits=bits)), ctypes.byref(need)) == 0
        return need.value

    one = ask([(14336, 4096)])
    assert one >= 8 * 14336 * 4096 + 4 * 4096 * 4096
    assert ask([(14336, 4096)] * 3) == one                           # one after another in the same room
    assert one < ask([(14336, 4096)], bits=32) < 2 * one
    assert ask([(1024, 256)] * 48) >= 48 * 8 * 1024 * 256 and ask([]) >= 256 and ask([(0, 5), (5, 0)]) >= 256
    assert ask([(256, 64)] * 3 + [(14336, 4096)]) == one
    need = ctypes.c_size_t(0)
    t = tensor(rows=1024, cols=256)
    assert lib.sffn_muon_workspace_bytes(ctypes.byref(t), 1, ctypes.byref(ns()), ctypes.byref(need)) == 0 and need.value >= 8 * 1024 * 256
    with_copy = need.value
    t.master = None                                                 # products of one term then
    assert lib.sffn_muon_workspace_bytes(ctypes.byref(t), 1, ctypes.byref(ns()), ctypes.byref(need)) == 0 and need.value != with_copy
    assert lib.sffn_muon_workspace_bytes(ctypes.byref(t), 1, ctypes.byref(ns()), None) == 1
