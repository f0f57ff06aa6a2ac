"""CPU-side check of the norms' backward pass: a workspace that lies over anything else of the call is refused."""
import ctypes

import pytest

from test_block_norm_abi import INVALID, at, call, grads, lib  # noqa: F401

# y, both gains, gate, h, stats; dh, dn, and every gradient
READ, WRITTEN = (0, 2, 3, 4, 5, 7, 8, 9), (10, 11, 12, 13, 14)


@pytest.mark.parametrize("n", READ + WRITTEN)
def test_a_workspace_over_another_array(lib, n):  # noqa: F811
    for shift in (0, 16, 32):
        assert lib.sffn_block_norm_backward(ctypes.byref(call()), ctypes.byref(grads(workspace=at(n) + shift)), None) == INVALID, shift
    need = ctypes.c_size_t(0)
    assert lib.sffn_block_norm_workspace_bytes(64, ctypes.byref(need)) == 0
    last = (need.value - 16) // 16 * 16  # its last bytes
    assert lib.sffn_block_norm_backward(ctypes.byref(call()), ctypes.byref(grads(workspace=at(n) - last)), None) == INVALID


def test_a_gate_of_channels_or_tokens(lib):  # noqa: F811
    for kind in (1, 2):
        for n in (4, 14):
            assert lib.sffn_block_norm_backward(ctypes.byref(call(gate_kind=kind)), ctypes.byref(grads(workspace=at(n))), None) == INVALID, (kind, n)
