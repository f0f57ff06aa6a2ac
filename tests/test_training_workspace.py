"""The workspace that training calls ask for follows what they have to hold: the values between products, and pieces of tiles where a
product can have any."""
import ctypes

import pytest

from test_training_abi import lib  # noqa: F401


def need(lib, T, D, H, dtype, backward):  # noqa: F811
    n = ctypes.c_size_t(0)
    assert lib.sffn_train_workspace_bytes(T, D, H, dtype, backward, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("T,D,H,backward,values,most", [
    (64, 256, 1024, 0, 64 * 1024 * 2, 3 << 20),           # z and u: 8 tiles of 4 blocks; y: one of 16
    (64, 256, 1024, 1, 3 * 64 * 1024 * 2, 7 << 20),
    (1, 64, 40, 0, 80, 1 << 20), (5, 64, 40, 1, 3 * 5 * 80, 1 << 20),
    (5, 4096, 14336, 1, 3 * 5 * 14336 * 2, 84 << 20), (8192, 4096, 14336, 0, 8192 * 14336 * 2, (8192 * 14336 * 2) + (81 << 20))])
def test_bf16(lib, T, D, H, backward, values, most):  # noqa: F811
    assert values <= need(lib, T, D, H, 1, backward) <= most


def test_bf16_grows_with_the_tokens(lib):  # noqa: F811
    """More tokens never need less: a buffer for a call's largest batch serves the smaller ones."""
    for backward in (0, 1):
        for D, H in ((64, 40), (256, 1024), (2048, 2045)):
            sizes = [need(lib, T, D, H, 1, backward) for T in list(range(0, 700, 7)) + [1000, 5000]]
            assert sizes == sorted(sizes)
