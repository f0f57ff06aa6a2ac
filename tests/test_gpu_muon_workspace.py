"""The workspace of the orthogonalised update and of the Muon step: what it held before does not matter, and what lies behind it keeps its marker, at sizes
whose tiles are whole, cut into pieces, joined in a cluster or by a launch of their own.  Run with `-m gpu` on a B200."""
import ctypes

import pytest
import torch

from test_gpu_muon import BF16, DEV, F32, gen, lib, normal  # noqa: F401
from test_muon_abi import Config, Orthogonal, Tensor, ns

pytestmark = pytest.mark.gpu
SHAPES = [((1, 1), 3), ((5, 700), 1), ((33, 70), 20), ((130, 260), 5), ((257, 300), 1), ((1000, 640), 1), ((256, 1024), 6), ((2049, 515), 1), ((300, 20000), 1),
          ((1300, 1290), 2), ((3000, 2100), 1), ((4100, 1030), 1)]


def pointer(t):
    return ctypes.c_void_p(t.data_ptr())


def workspaces(need):
    """Of exactly that size, full of zeros and full of NaN (in 16, 32 and 64 bits), with a marker behind."""
    for byte in (0, 0xff):
        room = torch.full((need + (1 << 20),), 0xa5, dtype=torch.uint8, device=DEV)
        room[:need] = byte
        assert room.data_ptr() % 256 == 0
        yield room


@pytest.mark.parametrize("bits", [16, 32])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("shape,n", SHAPES, ids=str)
def test_orthogonalize(lib, shape, n, dtype, bits):  # noqa: F811
    so, (R, C), g = lib.load_library(), shape, gen(shape[0])
    us = [normal(shape, g, 1e-2, dtype) for _ in range(n)]
    want = lib.orthogonalize(us, bits=bits)
    outs = [torch.empty_like(u) for u in us]
    items = (Orthogonal * n)(*[Orthogonal(pointer(u), C, pointer(o), C, R, C, int(dtype is BF16)) for u, o in zip(us, outs)])
    how, need = ns(bits=bits), ctypes.c_size_t(0)
    assert so.sffn_orthogonalize_workspace_bytes(items, n, ctypes.byref(how), ctypes.byref(need)) == 0
    status = torch.zeros(64, dtype=torch.int32, device=DEV)
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    for room in workspaces(need.value):
        assert so.sffn_orthogonalize(items, n, ctypes.byref(how), pointer(room), need, pointer(status), stream) == 0
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want)) and (room[need.value:] == 0xa5).all() and not status.any()
        for o in outs:
            o.fill_(7.0)


@pytest.mark.parametrize("kind", ["f32", "bf16", "master"])
@pytest.mark.parametrize("shape,n", [((33, 70), 20), ((257, 300), 3), ((256, 1024), 6), ((4100, 1030), 1)], ids=str)
def test_steps(lib, shape, n, kind):  # noqa: F811
    so, (R, C), g = lib.load_library(), shape, gen(shape[0])
    dtype = F32 if kind == "f32" else BF16
    start = [normal(shape, g, 0.1) for _ in range(n)]
    grads, moments = [normal(shape, g, 1e-3, dtype) for _ in range(n)], [normal(shape, g, 1e-3) for _ in range(n)]

    def fresh():
        return [w.to(dtype) for w in start], [m.clone() for m in moments], [w.clone() for w in start] if kind == "master" else [None] * n

    p, m, w = fresh()
    lib.muon_step(p, grads, [dict(m=t) for t in m], masters=w, lr=0.02, momentum=0.95, weight_decay=0.1, scale=1.0)
    status = torch.zeros(64, dtype=torch.int32, device=DEV)
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    config = Config(ns(), 0.95, 1, None, 0.0)
    need = ctypes.c_size_t(0)
    for turn in range(2):
        q, k, v = fresh()
        items = (Tensor * n)(*[Tensor(pointer(a), pointer(b), None if d is None else pointer(d), pointer(c), R, C, int(dtype is BF16), int(dtype is BF16), 0.02, 0.1, 1.0)
                               for a, b, c, d in zip(q, grads, k, v)])
        assert so.sffn_muon_workspace_bytes(items, n, ctypes.byref(config.ns), ctypes.byref(need)) == 0
        room = list(workspaces(need.value))[turn]
        assert so.sffn_muon_step(items, n, ctypes.byref(config), pointer(room), need, pointer(status), stream) == 0
        torch.cuda.synchronize()
        assert (room[need.value:] == 0xa5).all() and not status.any()
        for a, b in zip(q + k + [t for t in v if t is not None], p + m + [t for t in w if t is not None]):
            assert torch.equal(a, b)
