"""Outputs of the training calls that share memory with inputs or with each other are refused, before anything reaches a device."""
import ctypes

import pytest

from test_training_abi import Call, Grads, lib, vp  # noqa: F401

# T = 16, D = 64, H = 40, bf16: x, dy, y, dx 2 KB at rows of 128 bytes, z and u 1280 bytes at rows of 80, weights 5120 bytes.  Nothing is read.
PLACES = dict(x=0x100000, z=0x110000, u=0x118000, W_g=0x120000, W_up=0x130000, W_down=0x140000, b_g=0x150000, status=0x158000,
              workspace=0x10000000, dy=0x160000, y=0x170000, dx=0x180000, dW_g=0x190000, dW_up=0x1a0000, dW_down=0x1b0000, db_g=0x1c0000)


def forward(lib, ld=40, ld_y=64, T=16, **over):  # noqa: F811
    at = dict(PLACES, **over)
    c = Call(T, 64, 40, 1, 0, 3, at["x"], 64, at["W_g"], at["W_up"], at["W_down"], at["b_g"], at["z"], at["u"], ld, at["workspace"], 1 << 40, at["status"])
    return lib.gated_ffn_forward(ctypes.byref(c), vp(at["y"]), ctypes.c_int64(ld_y), None)


def backward(lib, ld=40, ld_dx=64, **over):  # noqa: F811
    at = dict(PLACES, **over)
    c = Call(16, 64, 40, 1, 0, 3, at["x"], 64, at["W_g"], at["W_up"], at["W_down"], None, at["z"], at["u"], ld, at["workspace"], 1 << 40, at["status"])
    g = Grads(at["dx"], ld_dx, at["dW_g"], at["dW_up"], at["dW_down"], at["db_g"])
    return lib.gated_ffn_backward(ctypes.byref(c), vp(at["dy"]), ctypes.c_int64(64), ctypes.byref(g), None)


@pytest.mark.parametrize("out,where", [
    ("z", "x"), ("u", "x"), ("y", "W_g"), ("y", "W_up"), ("y", "W_down"), ("z", "W_down"), ("u", "W_g"), ("y", "b_g"), ("z", "u"), ("z", "y"), ("u", "y"),
    ("y", "workspace"), ("u", "workspace")])
def test_outputs_of_the_forward_pass(lib, out, where):  # noqa: F811
    assert forward(lib, **{out: PLACES[where]}) == 1


@pytest.mark.parametrize("out", ["dW_g", "dW_up", "dW_down", "db_g"])
@pytest.mark.parametrize("where", ["x", "dy", "z", "u", "W_g", "W_up", "W_down", "workspace", "dx"])
def test_gradients_of_the_weights(lib, out, where):  # noqa: F811
    assert backward(lib, **{out: PLACES[where]}) == 1


@pytest.mark.parametrize("where", ["W_g", "W_up", "W_down", "dW_g", "dW_up", "dW_down", "db_g", "workspace"])
def test_dx(lib, where):  # noqa: F811
    assert backward(lib, dx=PLACES[where]) == 1


def test_edges(lib):  # noqa: F811
    """The last byte of one and the first of another, rows of one stride that start inside each other's, rows of two strides."""
    assert forward(lib, z=PLACES["x"] + 2048 - 16) == 1 and forward(lib, z=PLACES["x"] - 1280 + 16) == 1
    assert backward(lib, dW_g=PLACES["dy"] + 2048 - 16) == 1 and backward(lib, db_g=PLACES["dW_up"] + 5120 - 4) == 1
    assert forward(lib, ld=80, u=PLACES["z"] + 64) == 1                  # rows of 160 bytes, u's 80 from column 32 of z's 40
    assert forward(lib, ld=80, u=PLACES["z"] + 160 * 15 + 64) == 1       # only u's first row meets z's last one
    assert forward(lib, ld=80, u=PLACES["z"] - 160 * 15 - 64) == 1
    assert forward(lib, ld_y=128, y=PLACES["W_g"] - 256) == 1            # y's second row would lie in W_g
    assert forward(lib, ld=104, y=PLACES["z"] + 96) == 1                 # strides 208 and 128
