"""The workspace of the norms' backward pass: it may start on any 16 bytes, and what lies before and behind it keeps its marker.  Run with
`-m gpu` on a B200."""
import ctypes

import pytest
import torch

from test_block_norm_abi import Call, Grads
from test_gpu_block_norm import BF16, DEV, F32, inputs, lib  # noqa: F401

pytestmark = pytest.mark.gpu


ALL, MIXED = (F32, F32, F32), (BF16, F32, BF16)


@pytest.mark.parametrize("D,types", [(260, ALL)] + [(D, types) for D in (64, 264, 520, 1032, 2056, 4104, 8200, 16392) for types in (ALL, MIXED)],
                         ids=lambda v: {ALL: "f32", MIXED: "mixed"}.get(v, v))
@pytest.mark.parametrize("T", [1, 5, 700])
def test_starts_on_any_sixteen_bytes(lib, T, D, types):  # noqa: F811
    so = lib.load_library()
    c, dh, dn = inputs(T, D, types, "channel", True, True, seed=D)
    h, n, stats = lib.block_norm_forward(**c, n_dtype=types[2])
    want = lib.block_norm_backward(dh, dn, c["y"], h, stats, c["post_gain"], c["pre_gain"], c["gate"])
    need = ctypes.c_size_t(0)
    assert so.sffn_block_norm_workspace_bytes(D, ctypes.byref(need)) == 0
    p = lambda t: ctypes.c_void_p(t.data_ptr())  # noqa: E731
    code = lambda t: int(t is BF16)  # noqa: E731
    stream = ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    for offset in (0, 16, 32, 48):
        room = torch.full((need.value + 512,), 0xa5, dtype=torch.uint8, device=DEV)
        assert room.data_ptr() % 64 == 0
        out = {k: torch.empty_like(t) for k, t in want.items()}
        call = Call(T, D, *[code(t) for t in types], 1, p(c["y"]), D, None, 0, p(c["post_gain"]), p(c["pre_gain"]), p(c["gate"]), 0, 1.0, 0.0, p(h), D, None, 0, p(stats))
        grads = Grads(p(dh), D, p(dn), D, p(out["dy"]), D, p(out["dresid"]), D, p(out["dpost_gain"]), p(out["dpre_gain"]), p(out["dgate"]), 0,
                      ctypes.c_void_p(room.data_ptr() + offset), need.value)
        assert so.sffn_block_norm_backward(ctypes.byref(call), ctypes.byref(grads), stream) == 0
        torch.cuda.synchronize()
        for k in want:
            assert torch.equal(out[k], want[k]), (k, offset)
        assert (room[:offset] == 0xa5).all() and (room[offset + need.value:] == 0xa5).all()
